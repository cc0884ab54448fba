"""Token log probabilities where more logits than are kept come before the bound that the threads' maxima give: a higher bound is found among
those kept, and the logits are gone through again, as often as it takes."""
import math

import pytest
import torch

from paper_2503_09387_b200 import binding
from tests.test_gpu_operators import BF16, FP32, close, gen, ints

pytestmark = pytest.mark.gpu

VOCAB = 150000


def rows_of(dtype):
    """Rows whose best logits are in the hands of fewer threads than alternatives are asked for.  A thread reads every 512th vector of 16 bytes."""
    per = 4 if dtype is FP32 else 8
    i = torch.arange(VOCAB, device="cuda")
    noise = torch.randn(VOCAB, device="cuda", generator=gen(1)) * 0.1
    hot = (i // per) % 512 < 30
    return torch.stack([
        noise + torch.where(hot, 50.0, 0.0),                                # some 8800 of them: 1098 of a part of eight
        noise + torch.where(hot, 50.0 + i * 1e-4, 0.0),                     # ascending: every bound found is soon below the rest
        noise + torch.where(hot, 50.0 - i * 1e-4, 0.0),
        torch.where(hot, 50.0 + (i % 7).float(), noise),                    # seven values: a great many equal to the higher bound
        torch.where(hot, 50.0 + (i % 977).float() * 0.01, noise),
        torch.where((i // per) % 512 == 5, 50.0, 0.0) + noise]).to(dtype)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("copies", [1, 4, 20])                              # several CTAs a row, four, one
@pytest.mark.parametrize("top", [32, 31, 3])
def test_more_candidates_than_are_kept(top, copies, dtype):
    x = rows_of(dtype)
    tokens = ints([0, VOCAB - 1, 7, 20, 977, 41])
    n = x.shape[0]
    got = binding.token_logprobs(x.repeat(copies, 1), tokens.repeat(copies), top=top)
    order = torch.sort(x.float(), dim=-1, descending=True, stable=True)[1]
    rank = (order == tokens[:, None]).int().argmax(-1).int()
    logp = torch.log_softmax(x.double(), -1)
    entropy = -(logp.exp() * logp).sum(-1)
    # (as the other tests of these have it: differences to the maximum rounded once, 2^x to 2 units, the sums of a thread's logits)
    big = float(x.float().abs().max())
    rel = 2.0 ** -24 * (2 * big + 64) + 2.0 ** -22
    off, off_entropy = rel + 2.0 ** -22 * (big + 16), (rel + 2.0 ** -21) * (1 + math.log(VOCAB)) * entropy + 1e-30
    for c in range(copies):
        lp, h, place, best, best_lp = (t[c * n:(c + 1) * n] for t in got)
        assert torch.equal(place, rank) and torch.equal(best, order[:, :top].int())
        close(lp, logp.gather(1, tokens[:, None].long())[:, 0].cpu(), off)
        close(best_lp, logp.gather(1, order[:, :top]).cpu(), off)
        close(h, entropy.cpu(), off_entropy.cpu())
