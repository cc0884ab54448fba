"""What the stand-alone operators refuse, and the host-side pieces of them: no GPU is needed, since a call is checked before CUDA is
asked for anything."""
import ctypes as C

import pytest
import torch

from paper_2503_09387_b200 import binding, build
from tests import operators_reference as ref

P = 0x7f0000001000          # stands for a device pointer: no refused call looks at what it points to
INVALID, CAPACITY, UNSUPPORTED = binding.VS_ERR_INVALID_ARG, binding.VS_ERR_CAPACITY, binding.VS_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load_library()


def test_argument_blocks_match_the_header():
    assert C.sizeof(binding.VsCache) == 4 * 8 + 4 * 4
    assert binding.VS_ROPE.size == 3 * 8 + 5 * 8 + 8 + 12 * 4 and binding.VS_SCORES.size == 7 * 8 + 8 + 6 * 4
    seqs = 3 * 8 + 4 * 4
    assert binding.VS_CACHE_ROWS.size == seqs + 2 * 8 + 4 * 8 + 2 * 4 and binding.VS_CACHE_QUERIES.size == seqs + 5 * 8 + 4 * 8 + 6 * 4


ROPE = dict(x=P, out=P, pos=P, xr=128, xh=64, outr=128, outh=64, ps=3, theta=1e6, dtype=0, rows=3, heads=2, d=64, axes=2, il=0, inv=0, device=0,
            s0=20, s1=12, s2=0, s3=0)


@pytest.mark.parametrize("change,code", [
    (dict(x=0), INVALID), (dict(out=0), INVALID), (dict(pos=0), INVALID), (dict(x=P + 8), INVALID), (dict(out=P + 4), INVALID),
    (dict(pos=P + 4), INVALID), (dict(xr=132), INVALID), (dict(outh=65), INVALID), (dict(dtype=1, xh=66), INVALID), (dict(dtype=2), INVALID),
    (dict(rows=-1), INVALID), (dict(heads=0), INVALID), (dict(axes=0), INVALID), (dict(axes=5), INVALID), (dict(s1=11), INVALID),
    (dict(s0=33, s1=-1), INVALID), (dict(s0=2**31 - 1, s1=2**31 - 1), INVALID), (dict(theta=0.0), INVALID), (dict(theta=float("nan")), INVALID),
    (dict(theta=float("inf")), INVALID), (dict(d=40, s0=8), UNSUPPORTED), (dict(d=272, s0=124), UNSUPPORTED), (dict(d=0, s0=0, s1=0), UNSUPPORTED),
    (dict(heads=70000), UNSUPPORTED), (dict(rows=0, x=0), 0)])
def test_rope_axes_refusals(lib, change, code):
    assert lib.vs_rope_axes(binding.VS_ROPE.pack(*dict(ROPE, **change).values()), None) == code


CACHE = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=9, n_kv_heads=4, head_dim=128, device=0)
SEQS = dict(page_table=P, tokens=P, row_offsets=P, n_seqs=2, table_width=5, n_rows=7, reserved=0)
KV = dict(k=P, v=P, kr=512, kh=128, vr=512, vh=128, dtype=0, reserved=0)
QUERIES = dict(q=P, out=P, lse=P, ws=P, bytes=1 << 30, qr=3584, qh=128, outr=3584, outh=128, heads=28, causal=1, window=0, dtype=0, scale=0.1, reserved=0)
rows = lambda seqs={}, **kv: binding.VS_CACHE_ROWS.pack(*dict(SEQS, **seqs).values(), *dict(KV, **kv).values())
queries = lambda seqs={}, **q: binding.VS_CACHE_QUERIES.pack(*dict(SEQS, **seqs).values(), *dict(QUERIES, **q).values())


@pytest.mark.parametrize("cache,seqs,code", [
    (dict(), dict(n_seqs=0), INVALID), (dict(), dict(n_seqs=binding.VS_CACHE_MAX_SEQS + 1), CAPACITY), (dict(), dict(n_rows=-1), INVALID),
    (dict(), dict(row_offsets=0), INVALID),                          # seven rows of two sequences: not the same number each
    (dict(), dict(page_table=0), INVALID), (dict(), dict(tokens=0), INVALID), (dict(), dict(tokens=P + 2), INVALID),
    (dict(), dict(table_width=0), INVALID), (dict(k=None), dict(), INVALID), (dict(v_scale=None), dict(), INVALID), (dict(v=P + 8), dict(), INVALID),
    (dict(k_scale=P + 2), dict(), INVALID), (dict(n_pages=0), dict(), INVALID), (dict(n_kv_heads=0), dict(), INVALID),
    (dict(n_kv_heads=257), dict(), UNSUPPORTED), (dict(head_dim=96), dict(), UNSUPPORTED)])
def test_cache_refusals(lib, cache, seqs, code):
    c = binding.VsCache(**dict(CACHE, **cache))
    assert lib.vs_cache_write(c, rows(seqs), None) == lib.vs_cache_read(c, rows(seqs), None) == lib.vs_cache_attention(c, queries(seqs), None) == code


def test_cache_refusals_of_rows(lib):
    c = binding.VsCache(**CACHE)
    for f in (lib.vs_cache_write, lib.vs_cache_read):
        assert f(None, rows(), None) == f(c, None, None) == INVALID
        for change in (dict(k=0), dict(v=0), dict(k=P + 2), dict(kr=516), dict(vh=127), dict(dtype=2), dict(dtype=1, vh=130)):
            assert f(c, rows(**change), None) == INVALID, change
        assert f(c, rows(dict(n_rows=0), k=0, v=0), None) == 0


def test_cache_attention_refusals(lib):
    c, need = binding.VsCache(**CACHE), C.c_size_t(0)
    assert lib.vs_cache_attention_bytes(128, need) == 0 and need.value > 0
    assert lib.vs_cache_attention_bytes(96, need) == UNSUPPORTED and lib.vs_cache_attention_bytes(128, None) == INVALID
    lib.vs_cache_attention_bytes(128, need)
    assert lib.vs_cache_attention(None, queries(), None) == lib.vs_cache_attention(c, None, None) == INVALID
    for change, code in ((dict(q=0), INVALID), (dict(out=0), INVALID), (dict(ws=0), INVALID), (dict(bytes=need.value - 1), CAPACITY),
                         (dict(ws=P + 128), INVALID), (dict(q=P + 8), INVALID), (dict(qr=3588), INVALID), (dict(outr=3586), INVALID),
                         (dict(out=P + 4), INVALID), (dict(out=P + 8, dtype=1), INVALID), (dict(lse=P + 1), INVALID), (dict(heads=0), INVALID),
                         (dict(heads=30), UNSUPPORTED), (dict(heads=36), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
                         (dict(scale=float("inf")), INVALID), (dict(window=-1), INVALID), (dict(dtype=2), INVALID)):
        assert lib.vs_cache_attention(c, queries(**change), None) == code, change
    assert lib.vs_cache_attention(c, queries(dict(n_rows=1 << 28)), None) == UNSUPPORTED
    assert lib.vs_cache_attention(c, queries(dict(n_rows=0), q=0), None) == 0


def test_token_logprobs_refusals(lib):
    good = dict(logits=P, tokens=P, lp=P, entropy=P, rank=P, best=P, best_lp=P, stride=1000, dtype=1, rows=3, vocab=1000, top=5, device=0, reserved=0)
    for change, code in ((dict(logits=0), INVALID), (dict(logits=P + 2), INVALID), (dict(dtype=2), INVALID), (dict(rows=-1), INVALID),
                         (dict(vocab=0), INVALID), (dict(top=-1), INVALID), (dict(top=33), CAPACITY), (dict(vocab=4), INVALID), (dict(best=0), INVALID),
                         (dict(tokens=0), INVALID), (dict(tokens=P + 2), INVALID), (dict(lp=P + 2), INVALID), (dict(vocab=(1 << 30) + 1), UNSUPPORTED),
                         (dict(rows=(1 << 27) + 1), UNSUPPORTED), (dict(rows=0, logits=0), 0)):
        assert lib.vs_token_logprobs(binding.VS_SCORES.pack(*dict(good, **change).values()), None) == code, change
    assert lib.vs_token_logprobs(None, None) == INVALID


def test_binding_refuses_what_is_not_on_a_gpu():
    codes = torch.zeros((2, 1, 64, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.zeros((2, 1))
    with pytest.raises(ValueError):
        binding.PageCache(codes, codes, scales, scales)
    with pytest.raises(ValueError):
        binding.token_logprobs(torch.zeros((2, 9)), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.rope_axes(torch.zeros((2, 1, 64)), torch.zeros((1, 2), dtype=torch.int64), (32,))


def test_references_codes_are_the_formats():
    """nearest_code against every code's own value, every midpoint and its neighbours."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(ref.nearest_code(codes), codes)
    mid = (codes[1:] + codes[:-1]) / 2
    even = torch.where(torch.arange(126) % 2 == 0, codes[:-1], codes[1:])
    assert torch.equal(ref.nearest_code(mid), even) and torch.equal(ref.nearest_code(-mid), -even)
    assert torch.equal(ref.nearest_code(mid * (1 + 1e-9)), codes[1:]) and torch.equal(ref.nearest_code(mid * (1 - 1e-9)), codes[:-1])
    assert float(ref.nearest_code(torch.tensor([1e30], dtype=torch.float64))) == 448


def test_references_axes():
    assert ref.axes_of_pairs((2, 3, 1), False) == [0, 0, 1, 1, 1, 2]
    assert ref.axes_of_pairs((2, 3, 1), True) == [0, 1, 2, 0, 1, 1]


def test_refusals_of_outputs_over_inputs(lib):
    """In place means the same places."""
    assert lib.vs_rope_axes(binding.VS_ROPE.pack(*dict(ROPE, outr=256).values()), None) == INVALID
    assert lib.vs_rope_axes(binding.VS_ROPE.pack(*dict(ROPE, xh=128).values()), None) == INVALID
    c = binding.VsCache(**CACHE)
    for change in (dict(outh=256), dict(outr=128), dict(dtype=1)):
        assert lib.vs_cache_attention(c, queries(**change), None) == INVALID, change


def test_token_logprobs_of_no_rows(lib):
    """Nothing is asked for, whatever the number of alternatives: the outputs are empty and have no address."""
    none = dict(logits=0, tokens=0, lp=0, entropy=0, rank=0, best=0, best_lp=0, stride=1000, dtype=1, rows=0, vocab=1000, top=5, device=0, reserved=0)
    assert lib.vs_token_logprobs(binding.VS_SCORES.pack(*none.values()), None) == 0
    for change, code in ((dict(top=33), CAPACITY), (dict(vocab=4), INVALID), (dict(top=-1), INVALID)):
        assert lib.vs_token_logprobs(binding.VS_SCORES.pack(*dict(none, **change).values()), None) == code, change
