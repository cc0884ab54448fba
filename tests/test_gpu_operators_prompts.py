"""Attention over the paged cache for whole prompts: so many rows of a sequence that its tiles are more than the CTAs.  Every row against
the definition in 64 bits, over outputs that say which rows were never written."""
import pytest
import torch

from paper_2503_09387_b200 import binding
from tests import operators_reference as ref
from tests.test_gpu_operators import BF16, FP32, close, gen, ints, normal, offsets, tables

pytestmark = pytest.mark.gpu


def prompt_case(hkv, group, d, lengths, lens, causal=True, window=0, out_dtype=BF16):
    g = gen(sum(lens) + d + window)
    pages = sum((n + 63) // 64 for n in lengths) + 2
    cache = binding.PageCache.empty(pages, hkv, d)
    table = tables(g, lengths, pages)
    for i, n in enumerate(lengths):
        cache.write(table[i:i + 1], ints([0]), normal(g, n, hkv, d), normal(g, n, hkv, d, std=2.0))
    q = normal(g, sum(lens), hkv * group, d, std=1.2)
    out = torch.full((sum(lens) + 1, hkv * group, d), 77.0, dtype=out_dtype, device="cuda")
    lse = torch.full((sum(lens), hkv * group), 77.0, device="cuda")
    cache.attend(table, ints(lengths), q, out=out[:-1], lse=lse, row_offsets=offsets(lens) if len(lens) > 1 else None, causal=causal, window=window)
    left = int((lse == 77).sum())
    assert left == 0, f"{left} of {lse.numel()} rows and heads never written"
    o, l, o_off, l_off = ref.attend_at_once(cache, table, lengths, lens, q, d ** -0.5, causal, window)
    close(lse, l.cpu(), l_off.cpu(), "lse")
    close(out[:-1], o.cpu(), o_off.cpu(), "rows")
    assert cache.attend_status() == 0 and bool((out[-1] == 77).all())


@pytest.mark.parametrize("hkv,group,d,lengths,lens,causal,window", [
    (4, 7, 128, [5413], [5413], False, 0), (4, 7, 128, [5413], [5413], True, 1024), (4, 7, 128, [20000], [6000], False, 0),
    (4, 7, 128, [10533], [10533], True, 0), (4, 7, 128, [13440], [13440], True, 0), (1, 8, 128, [4737], [4737], False, 0),
    (1, 8, 64, [200], [9000], False, 0), (2, 8, 64, [9000], [9000], True, 200), (4, 4, 64, [300, 12000, 70], [1, 10001, 70], True, 1),
    (2, 7, 128, [6100, 6000], [5800, 5900], False, 0), (1, 1, 64, [40000], [40000], True, 130), (3, 7, 128, [9500], [5461], True, 0)])
def test_attend_prompts(hkv, group, d, lengths, lens, causal, window):
    prompt_case(hkv, group, d, lengths, lens, causal, window, FP32 if d == 64 else BF16)


def test_attend_a_prompt_is_its_chunks():
    """13440 causal rows (64 frames of 210 tokens) in one call and in calls of 1000: as far apart as two orders of the same sums."""
    g, n, hkv, group, d = gen(64), 13440, 4, 7, 128
    cache = binding.PageCache.empty(211, hkv, d)
    table = tables(g, [n], 211)
    cache.write(table, ints([0]), normal(g, n, hkv, d), normal(g, n, hkv, d, std=2.0))
    q = normal(g, n, hkv * group, d)
    out, lse = cache.attend(table, ints([n]), q, out_dtype=FP32)
    _, _, o_off, l_off = ref.attend_at_once(cache, table, [n], [n], q, d ** -0.5)
    for r in range(0, n, 1000):
        end = min(r + 1000, n)
        o, l = cache.attend(table, ints([end]), q[r:end], out_dtype=FP32)
        assert bool(((o - out[r:end]).abs() <= 2 * o_off[r:end] + 2.0 ** -22 * out[r:end].abs()).all())
        assert bool(((l - lse[r:end]).abs() <= 2 * l_off[r:end]).all())


def test_attend_time_of_many_rows_over_few_keys():
    """Four times the rows over 64 keys take about four times as long, not sixteen times: an item is not looked for from the first tile."""
    cache = binding.PageCache.empty(1, 4, 64)
    cache.write(ints([[0]]), ints([0]), normal(gen(1), 64, 4, 64), normal(gen(2), 64, 4, 64))

    def time_of(n):
        q = normal(gen(3), n, 32, 64)
        out, lse = torch.empty_like(q), torch.empty((n, 32), device="cuda")
        best = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            cache.attend(ints([[0]]), ints([64]), q, out=out, lse=lse, causal=False)
            b.record()
            torch.cuda.synchronize()
            best.append(a.elapsed_time(b))
        return min(best[1:])
    small, large = time_of(50000), time_of(200000)
    assert large < 8 * small, (small, large)
