"""Attention over pages whose values are zero or as small as the format goes: a row's sum and its lse have nothing to do with the values."""
import math

import pytest
import torch

from paper_2503_09387_b200 import binding
from tests import operators_reference as ref
from tests.test_gpu_operators import BF16, FP32, close, gen, ints, normal, tables

pytestmark = pytest.mark.gpu

WIDE = 1100            # a table so wide that calls of more than 32 packed rows go to the kernel for many rows


def scaled_pages(g, n, hkv, d, sizes, width=None):
    """A cache of n tokens, the values of page p times sizes(p)."""
    pages = (n + 63) // 64
    cache = binding.PageCache.empty(pages + 1, hkv, d)
    table = tables(g, [n], pages + 1, width)
    v = normal(g, n, hkv, d, dtype=FP32)
    for p in range(pages):
        v[64 * p:64 * p + 64] *= sizes(p)
    cache.write(table, ints([0]), normal(g, n, hkv, d, std=0.3, dtype=FP32), v)
    return cache, table


SIZES = {
    "zeros": lambda p: 0.0, "zeros first": lambda p: 0.0 if p < 1 else 1.0, "zeros last": lambda p: 0.0 if p > 0 else 1.0,
    "every second": lambda p: float(p % 2), "smallest": lambda p: 2.0 ** -112, "small and ordinary": lambda p: (2.0 ** -100, 1.0, 2.0 ** -109, 0.0)[p % 4],
    "both ends": lambda p: (0.0, 2.0 ** 118, 2.0 ** -112, 2.0 ** 60)[p % 4], "largest first": lambda p: 2.0 ** 118 if p == 0 else 0.0}


@pytest.mark.parametrize("what", list(SIZES))
@pytest.mark.parametrize("rows,hkv,group,d,n,width", [
    (1, 1, 7, 128, 128, None), (1, 1, 4, 64, 500, None), (2, 2, 7, 128, 1000, None), (40, 1, 7, 128, 300, None), (1, 4, 7, 128, 13504, None),
    (40, 1, 7, 128, 300, WIDE), (64, 1, 4, 64, 900, WIDE), (33, 4, 7, 128, 9000, None), (300, 2, 1, 128, 2500, WIDE)])
def test_attend_over_pages_of_zeros_and_extremes(rows, hkv, group, d, n, width, what):
    g = gen(rows + n)
    cache, table = scaled_pages(g, n, hkv, d, SIZES[what], width)
    q = normal(g, rows, hkv * group, d)
    for out_dtype in (BF16, FP32):
        out, lse = cache.attend(table, ints([n]), q, out_dtype=out_dtype)
        o, l, o_off, l_off = ref.attend_at_once(cache, table, [n], [rows], q, d ** -0.5)
        close(lse, l.cpu(), l_off.cpu(), "lse")
        close(out, o.cpu(), o_off.cpu(), "rows")
    assert cache.attend_status() == 0


@pytest.mark.parametrize("rows,width", [(1, None), (40, WIDE)])
def test_attend_zeros_beside_ordinary_values(rows, width):
    """128 equal keys, the first page's values zero: half of the second page's mean, and lse the logarithm of 128.  (Powers of two to 2^-22
    each, their sum, one division and product; the logarithm of that and its product with log 2.)"""
    cache = binding.PageCache.empty(2, 1, 128)
    v = torch.zeros(128, 1, 128, device="cuda")
    v[64:] = 2.0
    table = torch.full((1, width or 2), -1, dtype=torch.int32, device="cuda")
    table[0, :2] = ints([0, 1])
    cache.write(table, ints([0]), torch.zeros(128, 1, 128, device="cuda"), v)
    out, lse = cache.attend(table, ints([128]), normal(gen(1), rows, 7, 128), causal=False, out_dtype=FP32)
    assert float((out - 1.0).abs().max()) < 2.0 ** -20 and float((lse - math.log(128)).abs().max()) < 2e-6


@pytest.mark.parametrize("rows,n,width", [(1, 40, None), (1, 5000, None), (50, 200, WIDE)])
def test_attend_over_a_cache_that_was_never_written(rows, n, width):
    """PageCache.empty: every key and value zero."""
    cache = binding.PageCache.empty(100, 2, 64)
    table = torch.full((1, width or 100), -1, dtype=torch.int32, device="cuda")
    table[0, :100] = torch.arange(100, device="cuda")
    out, lse = cache.attend(table, ints([n]), normal(gen(2), rows, 8, 64), causal=False)
    assert bool((out == 0).all()) and float((lse - math.log(n)).abs().max()) < 1e-5


def test_rows_joined_by_their_lse():
    """A call over all keys and two calls over the halves, joined: the lse of a half of zeros is a number like any other."""
    g, n = gen(5), 2048
    cache, table = scaled_pages(g, n, 2, 128, lambda p: 0.0 if p < n // 128 else 1.0)
    q = normal(g, 3, 14, 128)
    whole, lse = cache.attend(table, ints([n]), q, causal=False, out_dtype=FP32)
    half = n // 128
    parts = [cache.attend(t.contiguous(), ints([n // 2]), q, causal=False, out_dtype=FP32) for t in (table[:, :half], table[:, half:2 * half])]
    l = torch.logaddexp(parts[0][1].double(), parts[1][1].double())
    o = sum(x.double() * (y.double() - l).exp()[..., None] for x, y in parts)
    assert float((l - lse).abs().max()) < 1e-4 and float((o - whole).abs().max()) < 1e-2


def test_read_of_the_largest_values():
    """What fp32 holds reads as the value of its code; codes of 256 and more at the largest scale stand for 2^128 and more."""
    cache = binding.PageCache.empty(1, 1, 64)
    x = torch.zeros(64, 1, 64, device="cuda")
    values = [3.4e38, -3.4e38, 3.2e38, 3.0e38, 1.7e38, math.inf, -math.inf, 1e30]
    x[0, 0, :8] = torch.tensor(values)
    cache.write(ints([[0]]), ints([0]), x, x * 2.0 ** -1)
    codes = cache.k.float()[0, 0, 0, :8]
    assert float(cache.k_scale[0, 0]) == 2.0 ** 120 and codes.tolist() == [256, -256, 240, 224, 128, 448, -448, 0]
    for dtype in (FP32, BF16):
        k, v = cache.read(ints([[0]]), ints([0]), torch.empty_like(x, dtype=dtype), torch.empty_like(x, dtype=dtype))
        assert k[0, 0, :8].tolist() == [math.inf, -math.inf, 240 * 2.0 ** 120, 224 * 2.0 ** 120, 2.0 ** 127, math.inf, -math.inf, 0]
        assert bool(torch.isfinite(v[0, 0, :5]).all())
