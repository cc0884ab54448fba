"""Attention over the paged cache where values are NaN: the rows that see such a token have NaN in its NaN dims, and no other row and no
other dim has anything of it, however the rows are worked on together."""
import pytest
import torch

from tests.test_gpu_operators import BF16, FP32, gen, ints, normal, offsets, pool, same_bits, tables

pytestmark = pytest.mark.gpu

WIDE = 1100            # a table so wide that calls of more than 32 packed rows go to the kernel for many rows


@pytest.mark.parametrize("out_dtype", [BF16, FP32])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 5), (True, 70), (False, 9), (False, 0)])
@pytest.mark.parametrize("hkv,group,d,lengths,lens,width", [
    (1, 4, 64, [40], [3], None), (2, 7, 128, [130], [4], None), (1, 7, 128, [300], [40], None), (2, 8, 64, [2000], [2], None),
    (1, 7, 128, [300], [40], WIDE), (2, 1, 128, [500, 200], [300, 33], WIDE), (1, 8, 64, [9000], [70], WIDE), (1, 3, 128, [64], [64], WIDE),
    (2, 7, 128, [7000, 900, 70], [40, 1, 6], WIDE), (4, 7, 128, [2000], [1400], None)])
def test_nan_values_reach_the_rows_that_see_them(hkv, group, d, lengths, lens, width, causal, window, out_dtype):
    g = gen(sum(lens) + d + window)
    pages = sum((n + 63) // 64 for n in lengths) + 1
    cache = pool(g, pages, hkv, d, junk=False)
    table = tables(g, lengths, pages, width)
    q = normal(g, sum(lens), hkv * group, d)
    off = offsets(lens) if len(lens) > 1 else None
    nan = torch.zeros((sum(lens), hkv, d), dtype=torch.bool)
    codes, places = cache.v.view(torch.uint8), []
    at = 0
    for i, (n, m) in enumerate(zip(lengths, lens)):
        # tokens that some rows see and some do not, the call's last one among them, and one that is seen by most or by none
        for token in {n - 1, n - 2, n - m + m // 2, n - m, max(n - m - 3, 0), n // 3, max(n - window - m // 2 - 1, 0)}:
            head, dim = token % hkv, (token * 37) % d
            places.append((int(table[i, token // 64]), head, token % 64, dim))
            for t in range(m):
                pos = n - m + t
                if (not causal or token <= pos) and (not window or token > pos - window):
                    nan[at + t, head, dim] = True
        at += m
    for p in places:
        codes[p] = 0
    want, lse = cache.attend(table, ints(lengths), q, row_offsets=off, causal=causal, window=window, out_dtype=out_dtype)
    for i, p in enumerate(places):
        codes[p] = 0x7f if i % 2 else 0xff
    out, lse2 = cache.attend(table, ints(lengths), q, row_offsets=off, causal=causal, window=window, out_dtype=out_dtype)
    where = nan.repeat_interleave(group, 1).cuda()
    assert torch.equal(torch.isnan(out), where) and not bool(torch.isnan(want).any())
    assert same_bits(out.masked_fill(where, 0), want.masked_fill(where, 0)) and same_bits(lse, lse2)
    assert cache.attend_status() == 0


@pytest.mark.parametrize("rows,width", [(3, None), (40, WIDE)])
def test_nan_keys_reach_the_rows_that_see_them(rows, width):
    g = gen(rows)
    cache = pool(g, 3, 1, 128, junk=False)
    table = tables(g, [150], 3, width)
    q = normal(g, rows, 7, 128)
    want, lse = cache.attend(table, ints([150]), q)
    cache.k.view(torch.uint8)[int(table[0, 2]), 0, 149 - 128, 5] = 0x7f
    out, lse2 = cache.attend(table, ints([150]), q)
    assert bool(torch.isnan(out[-1]).all()) and bool(torch.isnan(lse2[-1]).all())
    assert same_bits(out[:-1], want[:-1]) and same_bits(lse2[:-1], lse[:-1])
