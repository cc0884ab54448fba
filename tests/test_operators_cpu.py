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


def test_struct_layout_matches_header():
    assert C.sizeof(binding.VsCache) == 4 * 8 + 4 * 4 and C.sizeof(binding.VsCacheRows) == 3 * 8 + 4 * 4


ROPE = dict(x=P, xr=128, xh=64, out=P, outr=128, outh=64, dtype=0, rows=3, heads=2, d=64, pos=P, ps=3, axes=2, sections=(20, 12), il=0, inv=0,
            theta=1e6, device=0, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(pos=None), INVALID), (dict(sections=None), INVALID), (dict(x=P + 8), INVALID),
    (dict(out=P + 4), INVALID), (dict(pos=P + 4), INVALID), (dict(xr=132), INVALID), (dict(outh=65), INVALID), (dict(dtype=1, xh=66), INVALID),
    (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(heads=0), INVALID), (dict(axes=0), INVALID), (dict(axes=5), INVALID),
    (dict(sections=(20, 11)), INVALID), (dict(sections=(33, -1)), INVALID), (dict(sections=(2**31 - 1, 2**31 - 1)), INVALID),
    (dict(theta=0.0), INVALID), (dict(theta=float("nan")), INVALID), (dict(theta=float("inf")), INVALID), (dict(d=40, sections=(8, 12)), UNSUPPORTED),
    (dict(d=272, sections=(100, 36)), UNSUPPORTED), (dict(d=0, sections=(0, 0)), UNSUPPORTED), (dict(heads=70000), UNSUPPORTED),
    (dict(rows=0, x=None), 0)])
def test_rope_axes_refusals(lib, change, code):
    a = dict(ROPE, **change)
    sections = (C.c_int32 * 5)(*a["sections"]) if a["sections"] is not None else None
    assert lib.vs_rope_axes(a["x"], a["xr"], a["xh"], a["out"], a["outr"], a["outh"], a["dtype"], a["rows"], a["heads"], a["d"], a["pos"], a["ps"],
                            a["axes"], sections, a["il"], a["inv"], a["theta"], a["device"], a["stream"]) == code


CACHE = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=9, n_kv_heads=4, head_dim=128, device=0)
ROWS = dict(page_table=P, tokens=P, row_offsets=P, n_seqs=2, table_width=5, n_rows=7, reserved=0)
BAD = [(dict(), dict(n_seqs=0), INVALID), (dict(), dict(n_seqs=binding.VS_CACHE_MAX_SEQS + 1), CAPACITY), (dict(), dict(n_rows=-1), INVALID),
       (dict(), dict(row_offsets=None), INVALID),                     # seven rows of two sequences: not the same number each
       (dict(), dict(page_table=None), INVALID), (dict(), dict(tokens=None), INVALID), (dict(), dict(tokens=P + 2), INVALID),
       (dict(), dict(table_width=0), INVALID), (dict(k=None), dict(), INVALID), (dict(v_scale=None), dict(), INVALID), (dict(v=P + 8), dict(), INVALID),
       (dict(k_scale=P + 2), dict(), INVALID), (dict(n_pages=0), dict(), INVALID), (dict(n_kv_heads=0), dict(), INVALID),
       (dict(n_kv_heads=257), dict(), UNSUPPORTED), (dict(head_dim=96), dict(), UNSUPPORTED)]


@pytest.mark.parametrize("cache,rows,code", BAD)
def test_cache_refusals(lib, cache, rows, code):
    c, r = binding.VsCache(**dict(CACHE, **cache)), binding.VsCacheRows(**dict(ROWS, **rows))
    for f in (lib.vs_cache_write, lib.vs_cache_read):
        assert f(c, r, P, 512, 128, P, 512, 128, 0, None) == code
    assert lib.vs_cache_attention(c, r, P, 512, 128, 4, 0.1, 1, 0, P, 512, 128, 0, None, P, 1 << 30, None) == code


def test_cache_refusals_of_rows(lib):
    c, r = binding.VsCache(**CACHE), binding.VsCacheRows(**ROWS)
    for f in (lib.vs_cache_write, lib.vs_cache_read):
        for args in ((None, r, P, 512, 128, P, 512, 128, 0), (c, None, P, 512, 128, P, 512, 128, 0), (c, r, None, 512, 128, P, 512, 128, 0),
                     (c, r, P, 512, 128, None, 512, 128, 0), (c, r, P + 2, 512, 128, P, 512, 128, 0), (c, r, P, 516, 128, P, 512, 128, 0),
                     (c, r, P, 512, 128, P, 512, 127, 0), (c, r, P, 512, 128, P, 512, 128, 2), (c, r, P, 512, 128, P, 512, 130, 1)):
            assert f(*args, None) == INVALID
        assert f(c, binding.VsCacheRows(**dict(ROWS, n_rows=0)), None, 0, 0, None, 0, 0, 0, None) == 0


def test_cache_attention_refusals(lib):
    c, r, need = binding.VsCache(**CACHE), binding.VsCacheRows(**ROWS), C.c_size_t(0)
    assert lib.vs_cache_attention_bytes(128, need) == 0 and need.value > 0
    assert lib.vs_cache_attention_bytes(96, need) == UNSUPPORTED and lib.vs_cache_attention_bytes(128, None) == INVALID
    lib.vs_cache_attention_bytes(128, need)
    names = ("c", "r", "q", "qr", "qh", "heads", "scale", "causal", "window", "out", "outr", "outh", "dtype", "lse", "ws", "bytes")
    good = dict(zip(names, (c, r, P, 3584, 128, 28, 0.1, 1, 0, P, 3584, 128, 0, P, P, need.value)))
    for change, code in ((dict(q=None), INVALID), (dict(out=None), INVALID), (dict(ws=None), INVALID), (dict(bytes=need.value - 1), CAPACITY),
                         (dict(ws=P + 128), INVALID), (dict(q=P + 8), INVALID), (dict(qr=3588), INVALID), (dict(outr=3586), INVALID),
                         (dict(out=P + 4), INVALID), (dict(out=P + 8, dtype=1), INVALID), (dict(lse=P + 1), INVALID), (dict(heads=0), INVALID),
                         (dict(heads=30), UNSUPPORTED), (dict(heads=36), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
                         (dict(scale=float("inf")), INVALID), (dict(window=-1), INVALID), (dict(dtype=2), INVALID), (dict(c=None), INVALID),
                         (dict(r=binding.VsCacheRows(**dict(ROWS, n_rows=1 << 28))), UNSUPPORTED),
                         (dict(r=binding.VsCacheRows(**dict(ROWS, n_rows=0)), q=None), 0)):
        assert lib.vs_cache_attention(*dict(good, **change).values(), None) == code, change


def test_token_logprobs_refusals(lib):
    names = ("logits", "stride", "dtype", "rows", "vocab", "tokens", "top", "lp", "entropy", "rank", "best", "best_lp", "device")
    good = dict(zip(names, (P, 1000, 1, 3, 1000, P, 5, P, P, P, P, P, 0)))
    for change, code in ((dict(logits=None), INVALID), (dict(logits=P + 2), INVALID), (dict(dtype=2), INVALID), (dict(rows=-1), INVALID),
                         (dict(vocab=0), INVALID), (dict(top=-1), INVALID), (dict(top=33), CAPACITY), (dict(vocab=4), INVALID), (dict(best=None), INVALID),
                         (dict(tokens=None), INVALID), (dict(tokens=P + 2), INVALID), (dict(lp=P + 2), INVALID), (dict(vocab=(1 << 30) + 1), UNSUPPORTED),
                         (dict(rows=(1 << 27) + 1), UNSUPPORTED), (dict(rows=0, logits=None), 0)):
        assert lib.vs_token_logprobs(*dict(good, **change).values(), None) == code, change


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
