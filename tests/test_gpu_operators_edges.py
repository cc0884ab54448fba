"""The stand-alone operators where calls meet: two streams and two graphs at once, shared pages, outputs over inputs, other devices, and
the sizes at which a kernel's cut of the work changes."""
import math

import pytest
import torch

from paper_2503_09387_b200 import binding
from tests import operators_reference as ref
from tests.test_gpu_operators import BF16, FP32, attend_case, check_scores, close, gen, ints, normal, offsets, pool, same_bits, tables

pytestmark = pytest.mark.gpu


# ---- rotary positions ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,heads,d", [(3, 37, 80), (2, 150, 64), (5, 200, 16), (3, 9, 256), (4, 45, 48), (1, 17, 128), (301, 1, 32)])
def test_rope_axes_heads_of_several_warps(rows, heads, d, dtype):
    g = gen(rows + heads)
    half = d // 2
    sections = (half - half // 3, half // 3)
    x = normal(g, rows, heads, d, dtype=dtype)
    pos = torch.randint(0, 5000, (2, rows), device="cuda", generator=g)
    guard = torch.full((rows + 2, heads, d), 5.0, dtype=dtype, device="cuda")
    got = binding.rope_axes(x, pos, sections, out=guard[1:-1])
    want, bound = ref.rope(x, pos, sections, 1.0e6, False, False)
    close(got, want, bound)
    assert bool((guard[0] == 5).all()) and bool((guard[-1] == 5).all())


def test_calls_for_a_device_that_is_not_there():
    g = gen(1)
    x, pos = normal(g, 2, 3, 64), torch.zeros((1, 2), dtype=torch.int64, device="cuda")
    block = binding.VS_ROPE.pack(x.data_ptr(), x.data_ptr(), pos.data_ptr(), 192, 64, 192, 64, 2, 1e6, 0, 2, 3, 64, 1, 0, 0, 99, 32, 0, 0, 0)
    before = torch.cuda.current_device()
    assert binding.load_library().vs_rope_axes(block, 0) == binding.VS_ERR_CUDA
    assert torch.cuda.current_device() == before
    assert torch.equal(binding.rope_axes(x, pos, (32,)), x)                  # the error is nobody else's


# ---- attention ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("hkv,group,d,lengths,lens,window", [
    (2, 4, 64, [20000, 1, 9000], [1, 1, 1], 0),          # every item a whole number of runs of more than the least pages
    (2, 8, 64, [9000], [64], 0), (1, 7, 128, [6000, 3000], [1, 1], 2500), (2, 7, 128, [2700], [33], 0),
    (8, 1, 64, [500] * 30, [1] * 30, 0), (8, 4, 64, [700] * 12, [9] * 12, 0),       # more items than runs: equal ones
    (1, 1, 64, [0, 0, 260], [3, 1, 2], 0), (1, 8, 64, [257, 64], [2, 60], 0)])
def test_attend_where_the_cut_changes(hkv, group, d, lengths, lens, window):
    attend_case(hkv, group, d, lengths, lens, window=window)


def test_attend_most_sequences():
    n = binding.VS_CACHE_MAX_SEQS
    lens = [i % 2 for i in range(n - 1)] + [20]
    attend_case(1, 1, 64, [(i * 5) % 40 + lens[i] for i in range(n)], lens, ragged=True)


def test_attend_shared_and_repeated_pages():
    """Pages that two sequences share, and one that a sequence names three times."""
    g = gen(4)
    for n_rows in (1, 50):
        cache = pool(g, 6, 2, 128, junk=False)
        table = ints([[0, 1, 2], [0, 1, 3], [4, 4, 4]])
        cache.write(table[:1], ints([0]), normal(g, 192, 2, 128), normal(g, 192, 2, 128))
        cache.write(ints([[4]]), ints([0]), normal(g, 64, 2, 128), normal(g, 64, 2, 128))
        want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
        q = normal(g, 3 * n_rows, 14, 128)
        out, lse = cache.attend(table, ints([190, 170, 192]), q)
        o, l, o_off, l_off = want.attend(table.tolist(), [190, 170, 192], [n_rows] * 3, q, 128 ** -0.5)
        close(out, o, o_off)
        close(lse, l, l_off)


def held(g, hkv, d, lengths):
    pages = sum((n + 63) // 64 for n in lengths) + 1
    cache = pool(g, pages, hkv, d)
    table = tables(g, lengths, pages)
    for i, n in enumerate(lengths):
        cache.write(table[i:i + 1], ints([0]), normal(g, n, hkv, d), normal(g, n, hkv, d))
    return cache, table


@pytest.mark.parametrize("lens", [[1, 1], [40, 40], [1, 40]])
def test_attend_in_the_place_of_the_query(lens):
    g = gen(6)
    cache, table = held(g, 2, 128, [5000, 700])
    q = normal(g, sum(lens), 14, 128)
    out, lse = cache.attend(table, ints([5000, 700]), q, row_offsets=offsets(lens))
    same, lse2 = cache.attend(table, ints([5000, 700]), q, out=q, row_offsets=offsets(lens))
    assert same is q and same_bits(q, out) and same_bits(lse, lse2)
    for wrong in (q.transpose(0, 1).contiguous().transpose(0, 1), None):
        with pytest.raises(RuntimeError):
            if wrong is None:                                               # fp32 over bf16
                wide = torch.empty((sum(lens), 14, 256), dtype=BF16, device="cuda")
                cache.attend(table, ints([5000, 700]), wide[:, :, :128], out=wide.view(FP32), row_offsets=offsets(lens))
            else:
                cache.attend(table, ints([5000, 700]), q, out=q.as_strided(q.shape, wrong.stride()), row_offsets=offsets(lens))


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_on_two_streams_at_once(rows):
    g = gen(rows)
    cache, table = held(g, 4, 128, [6000, 3000])
    lengths = [ints([6000, 3000]), ints([3000, 5000])]
    tabs = [table, table.flip(0).contiguous()]
    lengths[1] = ints([2900, 5900])
    qs = [normal(g, 2 * rows, 28, 128) for _ in range(2)]
    want = [cache.attend(t, n, q) for t, n, q in zip(tabs, lengths, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(cache.attend(tabs[i], lengths[i], qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert same_bits(out, want[i][0]) and same_bits(lse, want[i][1])
    assert cache.attend_status() == 0


@pytest.mark.parametrize("rows", [1, 40])
def test_two_graphs_of_one_cache_side_by_side(rows):
    """Each graph has a workspace of its own, though both were captured on one stream that the cache had been used on."""
    g = gen(rows + 1)
    cache, table = held(g, 4, 128, [6000, 3000])
    lengths = [ints([6000, 3000]), ints([5000, 64])]
    qs = [normal(g, 2 * rows, 28, 128) for _ in range(2)]
    want = [cache.attend(table, n, q) for n, q in zip(lengths, qs)]
    on = torch.cuda.Stream()
    on.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(on):
        cache.attend(table, lengths[0], qs[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=on):
            first = cache.attend(table, lengths[i], qs[i])
            outs.append((first, cache.attend(table, lengths[i], qs[i])))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in outs[i]:
            assert same_bits(out, want[i][0]) and same_bits(lse, want[i][1])


def test_rows_behind_the_last_sequence_stay():
    g = gen(8)
    for lens in ([2, 1], [30, 7]):
        cache, table = held(g, 2, 64, [300, 200])
        n, off = sum(lens) + 3, offsets(lens)
        codes = cache.k.view(torch.uint8).clone()
        q = normal(g, n, 8, 64)
        out, lse = torch.full((n, 8, 64), 3.0, dtype=BF16, device="cuda"), torch.full((n, 8), 3.0, device="cuda")
        cache.attend(table, ints([300, 200]), q, out=out, lse=lse, row_offsets=off)
        assert bool((out[-3:] == 3).all()) and bool((lse[-3:] == 3).all()) and bool((lse[:-3] != 3).all())
        k, v = (torch.full((n, 2, 64), 3.0, device="cuda") for _ in range(2))
        cache.read(table, ints([0, 10]), k, v, row_offsets=off)
        assert bool((k[-3:] == 3).all()) and bool((v[-3:] == 3).all())
        assert torch.equal(cache.k.view(torch.uint8), codes)
        rows = normal(g, n, 2, 64)
        rows[-3:] = math.nan
        cache.write(table, ints([300 - lens[0], 200 - lens[1]]), rows, rows, row_offsets=off)
        k, v = (torch.zeros((n, 2, 64), device="cuda") for _ in range(2))
        cache.read(table, ints([300 - lens[0], 200 - lens[1]]), k, v, row_offsets=off)
        assert not bool(torch.isnan(k).any()) and bool((k[-3:] == 0).all())


# ---- token log probabilities -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,vocab", [(2, 140000), (9, 70001), (20, 66000), (76, 66000), (3, 32768), (3, 32772), (2, 8192), (2, 8193), (300, 260)])
def test_token_logprobs_parts_of_a_row(rows, vocab, dtype):
    """One to eight CTAs a row, whole steps of a CTA and ragged ones; some rows mostly -inf, tokens among them."""
    g = gen(rows + vocab)
    x = normal(g, rows, vocab, std=2.0, dtype=FP32)
    x[1::2] = torch.where(torch.rand((rows // 2, vocab), device="cuda", generator=g) < 0.999, -math.inf, x[1::2])
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    tokens[::3] = vocab - 1
    check_scores(x.to(dtype), tokens, 20)


@pytest.mark.parametrize("vocab", [999, 140000])
def test_token_logprobs_rows_at_the_ends_of_the_type(vocab):
    big = torch.finfo(FP32).max
    i = torch.arange(vocab, device="cuda")
    noise = normal(gen(2), vocab, dtype=FP32)
    some = (i * 7919) % vocab < vocab // 3
    for x, token in ((torch.where(some, big, -math.inf), 0), (torch.full((vocab,), big, device="cuda"), vocab - 1),
                     (torch.full((vocab,), -big, device="cuda"), 5), (torch.where(some, -big, -math.inf), 3),
                     (noise * 1e-40, 77), (torch.where(some, noise, -big), 2), (torch.where(some, noise, math.nan), vocab // 2),
                     (torch.where(i % 300 == 7, math.inf, noise), 307), (torch.full((vocab,), math.nan, device="cuda"), 4)):
        for k in (1, 32):
            check_scores(x[None].contiguous(), ints([token]), k)


def test_token_logprobs_where_another_type_is_the_default():
    x = normal(gen(3), 5, 700, dtype=FP32)
    want = binding.token_logprobs(x, ints([0, 1, 2, 3, 4]), top=3)
    torch.set_default_dtype(BF16)
    try:
        got = binding.token_logprobs(x, ints([0, 1, 2, 3, 4]), top=3)
    finally:
        torch.set_default_dtype(FP32)
    assert all(a.dtype is b.dtype and torch.equal(a, b) for a, b in zip(got, want))


# ---- the kernel for many rows: a table so wide that the calls above reach it whatever their rows and tokens ------------------------
WIDE = 1100


@pytest.mark.parametrize("out_dtype", [BF16, FP32])
@pytest.mark.parametrize("hkv,group,d,lengths,lens", [
    (2, 7, 128, [150, 33], [5, 5]), (1, 4, 64, [64, 64, 300], [9, 64, 17]), (2, 1, 128, [500], [33]), (1, 7, 128, [170], [170]),
    (2, 2, 64, [130, 5, 0, 260], [130, 5, 0, 100]), (1, 8, 128, [400], [37]), (1, 5, 64, [77, 900], [3, 60]), (1, 8, 64, [1, 65], [40, 33])])
def test_attend_many_rows(hkv, group, d, lengths, lens, out_dtype):
    attend_case(hkv, group, d, lengths, lens, out_dtype=out_dtype, width=WIDE)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 64), (True, 100), (False, 90), (True, 2**31 - 1)])
@pytest.mark.parametrize("lengths,lens", [([300], [40]), ([65, 200, 3], [10, 70, 7])])
def test_attend_many_rows_masks(lengths, lens, causal, window):
    attend_case(1, 7, 128, lengths, lens, causal=causal, window=window, width=WIDE)


def test_attend_many_rows_that_see_nothing():
    lens = [40, 50, 20]
    _, _, _, out, lse = attend_case(2, 7, 128, [0, 5, 190], lens, holes=[(2, 0), (2, 2)], ragged=True, width=WIDE)
    assert bool((out[:40] == 0).all()) and bool((lse[:40] == -math.inf).all())


def test_attend_many_rows_large_scores_unequal_pages_and_nan():
    attend_case(1, 7, 128, [500], [33], q_std=60.0, width=WIDE)
    g = gen(30)
    cache = pool(g, 6, 1, 128)
    table = tables(g, [384], 6, WIDE)
    k, v = normal(g, 384, 1, 128, dtype=FP32), normal(g, 384, 1, 128, dtype=FP32)
    for p, e in enumerate((0, 40, -60, 10, -100, 3)):
        v[64 * p:64 * p + 64] *= 2.0 ** e
        k[64 * p:64 * p + 64] *= 2.0 ** (-3 * p)
    cache.write(table, ints([0]), k, v)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    q = normal(g, 30, 4, 128)
    out, lse = cache.attend(table, ints([384]), q, out_dtype=FP32)
    o, l, o_off, l_off = want.attend(table.tolist(), [384], [30], q, 128 ** -0.5)
    close(out, o, o_off)
    close(lse, l, l_off)
    bad = q.clone()
    bad[0, 1, 5], bad[1, 2, 7] = math.nan, math.inf
    got, lse2 = cache.attend(table, ints([384]), bad, out_dtype=FP32)
    assert bool(torch.isnan(got[0, 1]).all()) and bool(torch.isnan(got[1, 2]).all()) and bool(torch.isnan(lse2[0, 1]))
    keep = torch.ones(30, 4, dtype=torch.bool)
    keep[0, 1] = keep[1, 2] = False
    assert torch.equal(got[keep.cuda()], out[keep.cuda()])


@pytest.mark.parametrize("hkv,group,d,lengths,lens", [
    (8, 8, 64, [70] * 20, [40] * 20), (4, 7, 128, [30] * 24, [12] * 24), (2, 7, 128, [5, 700, 64] * 6, [5, 1, 30] * 6), (8, 1, 128, [130] * 40, [70] * 40)])
def test_attend_more_items_than_ctas(hkv, group, d, lengths, lens):
    attend_case(hkv, group, d, lengths, lens)
    attend_case(hkv, group, d, lengths, lens, width=WIDE)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,vocab", [(9, 70003), (80, 9001), (3, 140001), (2, 5)])
def test_token_logprobs_rows_off_the_boundaries(rows, vocab, dtype):
    """Rows side by side of an odd size, and inside a wider tensor: first vectors in part ahead of the row, -inf among them and as the token's."""
    g = gen(vocab)
    for first, width in ((0, vocab), (1, vocab + 3), (3, vocab + 6)):
        wide = torch.full((rows, width), 1e30, device="cuda")
        x = normal(g, rows, vocab, std=2.0, dtype=FP32)
        x[::2, : vocab // 2] = -math.inf
        x[1::4] = -math.inf
        wide[:, first:first + vocab] = x
        tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
        tokens[::3] = vocab // 2 - 1
        tokens[1::3] = min(vocab - 1, 9)
        for top in (0, min(20, vocab)):
            check_scores(wide.to(dtype)[:, first:first + vocab], tokens, top)
