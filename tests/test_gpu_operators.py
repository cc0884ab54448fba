"""The stand-alone operators on the GPU against their definitions in 64 bits: rotary positions with several axes, the paged
8-bit cache and the attention over it, token log probabilities."""
import math

import pytest
import torch

from paper_2503_09387_b200 import binding
from tests import operators_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=BF16):
    return (torch.randn(shape, device="cuda", generator=g) * std).to(dtype)


def close(got, want, bound, what=""):
    """|got - want| <= bound + half a step of got's type, infinities and NaN in the same places."""
    got_, want = got.detach().cpu().double(), want.double()
    same = (got_ == want) | (torch.isnan(got_) & torch.isnan(want))
    over = (got_ - want).abs() - bound - ref.HALF_STEP[got.dtype] * want.abs() - 2.0 ** -133
    bad = ~same & ~(over <= 0)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float(over[bad].max()):.3g} (of {float(want[bad].abs().max()):.3g})"


# ---- rotary positions ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,heads,d,sections,interleaved", [
    (1, 32, 128, (16, 24, 24), False), (1, 1, 16, (8,), False), (7, 5, 64, (8, 12, 12), True), (65, 3, 80, (16, 12, 12), False),
    (33, 2, 256, (43, 1, 0, 84), True), (130, 20, 64, (32,), True), (2, 40, 96, (0, 24, 24), False), (5, 70, 128, (22, 21, 21), True)])
def test_rope_axes(rows, heads, d, sections, interleaved, dtype):
    g = gen(rows + d)
    x = normal(g, rows, heads, d, dtype=dtype)
    pos = torch.randint(0, 40000, (len(sections), rows), device="cuda", generator=g)
    for inverse in (False, True):
        got = binding.rope_axes(x, pos, sections, interleaved=interleaved, inverse=inverse)
        want, bound = ref.rope(x, pos, sections, 1.0e6, interleaved, inverse)
        close(got, want, bound, f"inverse={inverse}")


def test_rope_axes_far_and_negative_positions_and_other_bases():
    g = gen(3)
    x = normal(g, 9, 4, 128, dtype=FP32)
    pos = torch.tensor([[0, 1, -1, 2**31 - 1, -2**31 + 1, 123456789, 2**31 - 7, 3, 2**24 + 1]], device="cuda").repeat(2, 1)
    pos[1] = pos[1].flip(0)
    for theta in (1.0e6, 10000.0, 1.0, 0.5):
        want, bound = ref.rope(x, pos, (40, 24), theta, True, False)
        if theta < 1:
            bound = bound + 1e-3                       # angles far beyond 2^31
        close(binding.rope_axes(x, pos, (40, 24), theta=theta, interleaved=True), want, bound, f"theta={theta}")


def test_rope_axes_in_place_on_a_projections_rows():
    g = gen(4)
    qkv = normal(g, 19, 36 * 128)
    before = qkv.clone()
    x = qkv[:, :32 * 128].unflatten(1, (32, 128))
    pos = torch.randint(0, 9000, (3, 19), device="cuda", generator=g)
    want, bound = ref.rope(x, pos, (16, 24, 24), 1.0e6, False, False)
    assert binding.rope_axes(x, pos, (16, 24, 24), out=x) is x
    close(x, want, bound)
    assert torch.equal(qkv[:, 32 * 128:], before[:, 32 * 128:])        # the values' columns are not the heads'
    # heads and rows in any order, positions a view
    y = normal(g, 6, 11, 64, dtype=FP32).transpose(0, 1)
    wide = torch.randint(0, 100, (2, 40), device="cuda", generator=g)
    got = binding.rope_axes(y, wide[:, 3:14], (20, 12))
    want, bound = ref.rope(y, wide[:, 3:14], (20, 12), 1.0e6, False, False)
    close(got, want, bound)


def test_rope_axes_gradient_is_the_inverse():
    g = gen(5)
    x, up = normal(g, 3, 2, 32, dtype=FP32), normal(g, 3, 2, 32, dtype=FP32)
    pos = torch.randint(0, 500, (2, 3), device="cuda", generator=g)
    grad = binding.rope_axes(up, pos, (9, 7), inverse=True).cpu().double()
    # by differences of the 64-bit definition: the operator is linear, so any step will do
    f = lambda t: float((ref.rope(t, pos, (9, 7), 1.0e6, False, False)[0] * up.cpu().double()).sum())
    xd = x.cpu().double()
    for at in [(0, 0, 0), (1, 1, 15), (2, 0, 16), (2, 1, 31)]:
        hi, lo = xd.clone(), xd.clone()
        hi[at] += 0.5
        lo[at] -= 0.5
        assert abs(float(grad[at]) - (f(hi) - f(lo))) < 1e-5
    # the whole gradient by the formula, and there and back again
    want, bound = ref.rope(up, pos, (9, 7), 1.0e6, False, True)
    close(binding.rope_axes(up, pos, (9, 7), inverse=True), want, bound)
    back = binding.rope_axes(binding.rope_axes(x, pos, (9, 7)), pos, (9, 7), inverse=True)
    close(back, x.cpu().double(), 2 * ref.rope(x, pos, (9, 7), 1.0e6, False, False)[1].abs() + 2.0 ** -22)


def test_rope_axes_no_rows():
    x = torch.empty((0, 4, 64), dtype=BF16, device="cuda")
    assert binding.rope_axes(x, torch.empty((1, 0), dtype=torch.int64, device="cuda"), (32,)).shape == (0, 4, 64)


# ---- the paged cache -----------------------------------------------------------------------------------------------
def pool(g, n_pages, hkv, d, junk=True):
    """A cache whose every byte holds something: any code at all where `junk` (NaN among them), scales of all sizes."""
    codes = lambda: torch.randint(0, 256, (n_pages, hkv, 64, d), device="cuda", generator=g, dtype=torch.uint8)
    scales = lambda: torch.exp2(torch.randint(-9, -3, (n_pages, hkv), device="cuda", generator=g).float())
    k, v = codes(), codes()
    if not junk:
        for t in (k, v):
            t[(t & 127) == 127] = 5
    return binding.PageCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), scales(), scales())


def tables(g, lengths, n_pages, width=None):
    need = [(n + 63) // 64 for n in lengths]
    order = torch.randperm(n_pages, device="cuda", generator=g).int()
    table = torch.full((len(lengths), width or max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    assert at <= n_pages
    return table


def same_bits(a, b):
    """Equal as they are stored, NaN included."""
    kind = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets(lens):
    return ints([0] + list(torch.tensor(lens).cumsum(0)))


def same_cache(cache, want, what=""):
    for name, got, codes in (("k", cache.k, want.codes[0]), ("v", cache.v, want.codes[1])):
        got = got.cpu().float().double()
        assert bool(((got == codes) | (torch.isnan(got) & torch.isnan(codes))).all()), f"{what} {name} codes"
    assert torch.equal(cache.k_scale.cpu().double(), want.scale[0]) and torch.equal(cache.v_scale.cpu().double(), want.scale[1]), f"{what} scales"


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hkv,d,start,lens", [
    (4, 128, [0], [1]), (4, 128, [63], [2]), (2, 64, [0, 5, 64, 127], [64, 59, 65, 1]), (1, 128, [17, 0, 200], [300, 0, 1]),
    (3, 64, [1, 2, 3, 4, 5, 6, 7, 8, 9], [1, 1, 1, 1, 1, 1, 1, 1, 1]), (8, 128, [40, 0], [130, 64])])
def test_cache_write_and_read(hkv, d, start, lens, dtype):
    g = gen(sum(lens) + d)
    n, pages = sum(lens), sum((s + m + 63) // 64 for s, m in zip(start, lens)) + 2
    cache = pool(g, pages, hkv, d)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    table = tables(g, [s + m for s, m in zip(start, lens)], pages)
    k, v = normal(g, n, hkv, d, dtype=dtype), normal(g, n, hkv, d, std=3.0, dtype=dtype)
    k[::5] *= 37.0
    v[::7] *= 1000.0
    off = None if len(set(lens)) == 1 else offsets(lens)
    cache.write(table, ints(start), k, v, row_offsets=off)
    want.write(table.tolist(), start, lens, k, v)
    same_cache(cache, want)
    for out_dtype in (BF16, FP32):
        ko, vo = torch.full((n, hkv, d), 7.0, dtype=out_dtype, device="cuda"), torch.full((n, hkv, d), 7.0, dtype=out_dtype, device="cuda")
        cache.read(table, ints(start), ko, vo, row_offsets=off)
        at = 0
        for i, (s, m) in enumerate(zip(start, lens)):
            for got, which in ((ko, 0), (vo, 1)):
                assert torch.equal(got[at:at + m].cpu().double(), want.rows(which, table.tolist(), i, s, s + m)[0])
            at += m


def test_cache_written_token_by_token_with_growing_scales():
    g = gen(11)
    cache = pool(g, 5, 2, 64)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    table = tables(g, [140, 70], 5)
    for t in range(140):
        seqs = [t, min(t, 69)]
        k, v = normal(g, 2, 2, 64, std=2.0 ** (t % 23 - 11)), normal(g, 2, 2, 64, std=1.0 + t)
        if t < 70:
            cache.write(table, ints(seqs), k, v)
            want.write(table.tolist(), seqs, [1, 1], k, v)
        else:
            cache.write(table[:1], ints(seqs[:1]), k[:1], v[:1])
            want.write(table[:1].tolist(), seqs[:1], [1], k[:1], v[:1])
    same_cache(cache, want)


def test_cache_write_of_unusual_values():
    """Zeros, the smallest and largest numbers, infinities, NaN; borders of the format and ties."""
    cache = pool(gen(1), 4, 1, 64)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    k = torch.zeros((4 * 64, 1, 64), device="cuda")
    v = torch.zeros_like(k)
    k[64:128] = 3.4e38
    k[70, 0, 3] = -3.4e38
    k[128:192] = 1e-45
    k[192:256] = 1e-33 * torch.randn(64, 1, 64, device="cuda", generator=gen(2))
    ties = torch.tensor([448.0, 464.0, 432.0, 1.0625, 1.1875, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 0.0068, -0.0, 447.9, 240.0, 248.0, 232.0])
    v[:64, 0, :16] = ties.cuda()
    v[0, 0, 1] = 448.0
    v[64:128, 0] = torch.linspace(-448, 448, 64, device="cuda")[:, None] * torch.linspace(0, 1, 64, device="cuda")
    v[130, 0, 5], v[131, 0, 6], v[132, 0, 7], v[133] = math.inf, -math.inf, math.nan, 2.5
    v[200:210] = math.nan
    table = ints([[2, 0, 3, 1]])
    cache.write(table, ints([0]), k, v)
    want.write(table.tolist(), [0], [256], k, v)
    same_cache(cache, want)
    ko, vo = cache.read(table, ints([0]), torch.empty_like(k), torch.empty_like(v))
    assert bool(torch.isnan(vo[132, 0, 7])) and float(vo[130, 0, 5]) == 448.0 * float(cache.v_scale[3, 0]) and float(ko[:64].abs().max()) == 0.0


def test_cache_rows_without_a_page():
    """Entries of the table that are no page, and places beyond it: nothing is written, zeros are read, other pages stay."""
    g = gen(21)
    cache = pool(g, 6, 2, 128)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    table = ints([[4, -1, 2], [0, 6, 2**31 - 1]])
    start, lens = [10, 30], [300, 170]
    k, v = normal(g, 470, 2, 128), normal(g, 470, 2, 128)
    cache.write(table, ints(start), k, v, row_offsets=offsets(lens))
    want.write(table.tolist(), start, lens, k, v)
    same_cache(cache, want)
    ko, vo = cache.read(table, ints(start), torch.full_like(k, 9.0), torch.full_like(v, 9.0), row_offsets=offsets(lens))
    assert torch.equal(vo[:300].cpu().double(), want.rows(1, table.tolist(), 0, 10, 310)[0])
    assert torch.equal(ko[300:].cpu().double(), want.rows(0, table.tolist(), 1, 30, 200)[0])


def test_cache_rows_as_columns_of_a_projection():
    g = gen(22)
    cache = pool(g, 4, 4, 128)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    qkv = normal(g, 100, 36 * 128)
    k, v = qkv[:, 28 * 128:32 * 128].unflatten(1, (4, 128)), qkv[:, 32 * 128:].unflatten(1, (4, 128))
    table = tables(g, [103], 4)
    cache.write(table, ints([3]), k, v)
    want.write(table.tolist(), [3], [100], k, v)
    same_cache(cache, want)
    keep = qkv.clone()
    cache.read(table, ints([3]), qkv[:, :4 * 128].unflatten(1, (4, 128)), qkv[:, 4 * 128:8 * 128].unflatten(1, (4, 128)))
    assert torch.equal(qkv[:, 8 * 128:], keep[:, 8 * 128:])
    assert torch.equal(qkv[:, :512].unflatten(1, (4, 128)).cpu().double(), want.rows(0, table.tolist(), 0, 3, 103)[0])


# ---- attention over the cache ----------------------------------------------------------------------------------------
def attend_case(hkv, group, d, lengths, lens, seed=0, causal=True, window=0, out_dtype=BF16, q_std=1.2, width=None, holes=(), ragged=None, junk_scale=False):
    g = gen(seed + sum(lens) * 7 + d)
    pages = sum((n + 63) // 64 for n in lengths) + 2
    cache = pool(g, pages, hkv, d)
    table = tables(g, lengths, pages, width)
    # tokens that exist: ordinary numbers; all that lies behind them in their pages stays what it was, NaN included
    for i, n in enumerate(lengths):
        if n:
            std = 1.0 if i % 2 == 0 else 0.3
            cache.write(table[i:i + 1], ints([0]), normal(g, n, hkv, d, std=std), normal(g, n, hkv, d, std=2.0))
    for i, p in holes:
        table[i, p] = -1
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    q = normal(g, sum(lens), hkv * group, d, std=q_std)
    scale = d ** -0.5
    off = offsets(lens) if (ragged or len(set(lens)) > 1) else None
    guard = torch.full((sum(lens) + 2, hkv * group, d), 77.0, dtype=out_dtype, device="cuda")
    out, lse = cache.attend(table, ints(lengths), q, out=guard[1:-1], row_offsets=off, causal=causal, window=window)
    o, l, o_off, l_off = want.attend(table.tolist(), lengths, lens, q, scale, causal, window)
    close(out, o, o_off, "rows")
    close(lse, l, l_off, "lse")
    assert cache.attend_status() == 0
    assert bool((guard[0] == 77).all()) and bool((guard[-1] == 77).all())
    return cache, table, q, out, lse


@pytest.mark.parametrize("group,d", [(7, 128), (4, 64), (1, 128), (8, 64), (3, 128)])
@pytest.mark.parametrize("lengths", [[1], [63], [64], [65], [700], [2, 0, 129, 1000, 64]])
def test_attend_one_token(group, d, lengths):
    attend_case(2, group, d, lengths, [1] * len(lengths))


@pytest.mark.parametrize("out_dtype", [BF16, FP32])
@pytest.mark.parametrize("hkv,group,d,lengths,lens", [
    (4, 7, 128, [200], [2]), (2, 7, 128, [150, 33], [5, 5]), (1, 4, 64, [64, 64, 300], [1, 64, 17]), (2, 1, 128, [500], [33]),
    (1, 7, 128, [170], [170]), (2, 2, 64, [130, 5, 0, 260], [130, 5, 0, 100]), (1, 8, 128, [400], [37]), (1, 5, 64, [77, 900], [3, 60])])
def test_attend_several_rows(hkv, group, d, lengths, lens, out_dtype):
    attend_case(hkv, group, d, lengths, lens, out_dtype=out_dtype)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 64), (True, 100), (False, 90), (True, 2**31 - 1)])
@pytest.mark.parametrize("lengths,lens", [([300], [1]), ([300], [40]), ([65, 200, 3], [1, 70, 3])])
def test_attend_masks(lengths, lens, causal, window):
    attend_case(1, 7, 128, lengths, lens, causal=causal, window=window)


@pytest.mark.parametrize("lens", [[1, 1, 1], [3, 9, 2], [40, 50, 20]])
def test_attend_rows_that_see_nothing(lens):
    """Sequences without tokens, rows ahead of a sequence's first token (more rows than tokens), pages that are not there."""
    _, _, _, out, lse = attend_case(2, 7, 128, [0, 5, 190], lens, holes=[(2, 0), (2, 2)], ragged=True)
    assert bool((out[:lens[0]] == 0).all()) and bool((lse[:lens[0]] == -math.inf).all())
    attend_case(1, 4, 64, [100, 130], [2, 2], holes=[(0, 0), (0, 1), (1, 2)])


def test_attend_large_scores_and_unequal_pages():
    """Scores of hundreds; pages whose scales differ by 2^40 and more, the largest values behind the smallest weights."""
    attend_case(1, 7, 128, [500], [1], q_std=60.0)
    attend_case(1, 7, 128, [500], [33], q_std=60.0)
    for rows in (1, 30):
        g = gen(rows)
        cache = pool(g, 6, 1, 128)
        table = tables(g, [384], 6)
        k, v = normal(g, 384, 1, 128, dtype=FP32), normal(g, 384, 1, 128, dtype=FP32)
        for p, e in enumerate((0, 40, -60, 10, -100, 3)):
            v[64 * p:64 * p + 64] *= 2.0 ** e
            k[64 * p:64 * p + 64] *= 2.0 ** (-3 * p)
        cache.write(table, ints([0]), k, v)
        want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
        q = normal(g, rows, 4, 128)
        out, lse = cache.attend(table, ints([384]), q, out_dtype=FP32)
        o, l, o_off, l_off = want.attend(table.tolist(), [384], [rows], q, 128 ** -0.5)
        close(out, o, o_off)
        close(lse, l, l_off)


def test_attend_nan_and_infinite_queries_stay_in_their_rows():
    for rows in (2, 40):
        g = gen(9)
        cache = pool(g, 4, 1, 128)
        table = tables(g, [200], 4)
        cache.write(table, ints([0]), normal(g, 200, 1, 128), normal(g, 200, 1, 128))
        q = normal(g, rows, 4, 128)
        clean = cache.attend(table, ints([200]), q)[0]
        bad = q.clone()
        bad[0, 1, 5], bad[1, 2, 7] = math.nan, math.inf
        out, lse = cache.attend(table, ints([200]), bad)
        assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(out[1, 2]).all()) and bool(torch.isnan(lse[0, 1]))
        keep = torch.ones(rows, 4, dtype=torch.bool)
        keep[0, 1] = keep[1, 2] = False
        assert torch.equal(out[keep.cuda()], clean[keep.cuda()])


def test_attend_strides_and_same_bits_every_time():
    g = gen(12)
    cache, table, q, out, lse = attend_case(2, 7, 128, [3000, 100, 900], [1, 1, 1], seed=5)
    wide = torch.zeros((3, 14 * 128 + 64), dtype=BF16, device="cuda")
    view = wide[:, 64:].unflatten(1, (14, 128))
    view.copy_(q)
    to = torch.zeros((14, 3, 128), dtype=BF16, device="cuda").transpose(0, 1)
    again, lse2 = cache.attend(table, ints([3000, 100, 900]), view, out=to)
    assert torch.equal(again, out) and torch.equal(lse, lse2)
    for _ in range(20):
        assert torch.equal(cache.attend(table, ints([3000, 100, 900]), q)[0], out)


def test_attend_many_sequences():
    lens = [1 + (i * 7) % 3 for i in range(200)]
    attend_case(1, 2, 64, [lens[i] + (i * 37) % 150 for i in range(200)], lens)


def test_cache_beyond_32_bits():
    """Pages whose codes lie more than 4 GiB into the pool."""
    n_pages = (1 << 32) // (64 * 128 * 4) + 40
    k = torch.zeros((n_pages, 4, 64, 128), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros((n_pages, 4, 64, 128), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    cache = binding.PageCache(k, v, torch.zeros((n_pages, 4), device="cuda"), torch.zeros((n_pages, 4), device="cuda"))
    g = gen(2)
    table = ints([[n_pages - 1, 3, n_pages - 20, n_pages - 2]])
    rows_k, rows_v = normal(g, 250, 4, 128), normal(g, 250, 4, 128)
    cache.write(table, ints([0]), rows_k, rows_v)
    small = binding.PageCache.empty(4, 4, 128)
    small.write(ints([[0, 1, 2, 3]]), ints([0]), rows_k, rows_v)
    picked = table[0].long()
    assert torch.equal(cache.k.view(torch.uint8)[picked], small.k.view(torch.uint8))
    for rows in (1, 30):
        q = normal(g, rows, 8, 128)
        assert torch.equal(cache.attend(table, ints([250]), q)[0], small.attend(ints([[0, 1, 2, 3]]), ints([250]), q)[0])
    a = cache.read(table, ints([0]), torch.empty_like(rows_k), torch.empty_like(rows_v))
    b = small.read(ints([[0, 1, 2, 3]]), ints([0]), torch.empty_like(rows_k), torch.empty_like(rows_v))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- token log probabilities -------------------------------------------------------------------------------------------
def check_scores(logits, tokens, top):
    got = [t.cpu() for t in binding.token_logprobs(logits, tokens, top=top)]
    want = ref.token_logprobs(logits, tokens, top)
    n = logits.shape[1]
    big = float(logits.float()[torch.isfinite(logits.float())].abs().max()) if bool(torch.isfinite(logits.float()).any()) else 0.0
    # differences to the maximum rounded once (2^-24 of them, a relative error of their exponentials), 2^x to 2 units, sums of up to n terms by
    # threads of a few hundred
    rel = 2.0 ** -24 * (2 * big + 64) + 2.0 ** -22
    for r, (lp, entropy, rank, best, best_lp) in enumerate(want):
        assert int(got[2][r]) == rank and got[3][r].tolist() == best, f"row {r}"
        close(got[0][r], torch.tensor(lp, dtype=torch.float64), rel + 2.0 ** -22 * (big + 16), f"logprob of row {r}")
        close(got[4][r], torch.tensor(best_lp, dtype=torch.float64), rel + 2.0 ** -22 * (big + 16), f"alternatives of row {r}")
        close(got[1][r], torch.tensor(entropy, dtype=torch.float64), 0 if entropy != entropy else (rel + 2.0 ** -21) * (1 + math.log(n)) * entropy + 1e-30, f"entropy of row {r}")


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 2, 0), (3, 31, 31), (2, 1000, 32), (1, 32000, 20), (5, 4099, 7), (200, 513, 3), (1, 152064, 32), (40, 9001, 1)])
def test_token_logprobs(rows, vocab, top, dtype):
    g = gen(vocab + rows)
    logits = normal(g, rows, vocab, std=3.0, dtype=dtype)
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    tokens[::3] = logits[::3].argmax(-1).int()
    check_scores(logits, tokens, top)


def test_token_logprobs_rows_that_begin_anywhere():
    g = gen(8)
    wide = normal(g, 4, 5003, std=2.0, dtype=FP32)
    check_scores(wide[:, 1:5000], ints([0, 4998, 17, 2500]), 9)
    check_scores(wide.bfloat16()[:, 3:4999], ints([0, 4995, 17, 2500]), 9)


def test_token_logprobs_ties_masks_and_unusual_rows():
    vocab = 20000
    x = torch.zeros((12, vocab), device="cuda")
    x[1] = -math.inf                                                        # no token can be
    x[2] = -math.inf
    x[2, [5, 19999, 700]] = torch.tensor([1.0, 1.0, 3.0], device="cuda")    # three can
    x[3] = normal(gen(1), vocab, dtype=FP32)
    x[3, 77] = math.nan
    x[4, 123] = math.inf
    x[5, 9] = 200.0                                                         # all but certain
    x[6] = torch.linspace(-5, 9, vocab, device="cuda")                      # ascending: every thread's last is its best
    x[7] = torch.linspace(9, -5, vocab, device="cuda")
    x[8] = torch.where(torch.arange(vocab, device="cuda") % 512 < 25, 4.0, -torch.arange(vocab, device="cuda").float() * 1e-4)
    x[9, ::2] = -0.0                                                        # equal to 0
    x[10] = -3.4e38
    x[10, 4000] = -3.3e38
    x[11, 3] = 16.0                                                         # certain but for what fp32 sums would lose
    tokens = ints([19999, 3, 700, 77, 5, 0, 19999, 0, 24, 1, 4000, 4])
    for top in (1, 20, 32):
        check_scores(x, tokens, top)
    check_scores(x[:3].bfloat16(), ints([-1, 20000, 19999]), 5)
    tall = x[:3].repeat(120, 1)                                              # many rows: a CTA a row
    check_scores(tall, ints([5, 6, 7] * 120), 20)


def test_token_logprobs_more_above_the_bound_than_are_kept():
    """The best logits in a few threads' hands: those of one thread come before everybody else's maximum."""
    vocab = 150000
    x = torch.randn(2, vocab, device="cuda", generator=gen(6)) * 0.1
    i = torch.arange(vocab, device="cuda")
    x[0] += torch.where((i // 4) % 512 < 20, 50.0, 0.0)
    x[1] += torch.where((i // 4) % 512 == 5, 50.0, 0.0)
    check_scores(x, ints([0, 20]), 32)
    check_scores(x.repeat(160, 1)[:3], ints([0, 20, 1]), 32)


def test_token_logprobs_without_tokens():
    x = normal(gen(2), 3, 999, dtype=FP32)
    lp, entropy, rank, best, best_lp = binding.token_logprobs(x, top=4)
    assert lp.tolist() == [0, 0, 0] and rank.tolist() == [-1, -1, -1] and torch.equal(best[:, 0].long(), x.argmax(-1))
    assert torch.equal(entropy, binding.token_logprobs(x, ints([0, 1, 2]))[1])


# ---- together --------------------------------------------------------------------------------------------------------
def step(qkv, pos, cache, table, start, hq, hkv, d):
    """A program's step: rotate the projected rows, append them, attend."""
    heads = qkv[:, :(hq + hkv) * d].unflatten(1, (hq + hkv, d))
    binding.rope_axes(heads, pos, (16, 24, 24), out=heads)
    n = qkv.shape[0] // table.shape[0]
    cache.write(table, start, heads[:, hq:], qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)))
    return cache.attend(table, start + n, heads[:, :hq])


def test_frames_then_answer_tokens():
    """Two streams, frames of different sizes, then answer tokens, on a stream of the program's own; against the definitions one after
    the other, the cache's codes among them; the last step's logits scored."""
    hq, hkv, d = 14, 2, 128
    g = gen(77)
    cache = pool(g, 14, hkv, d)
    want = ref.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale)
    table = tables(g, [400, 400], 14)
    start = [0, 0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for n in (50, 91, 1, 1, 3, 1):
            qkv = normal(g, 2 * n, (hq + 2 * hkv) * d)
            pos = torch.randint(0, 500, (3, 2 * n), device="cuda", generator=g)
            turned, bound = ref.rope(qkv[:, :(hq + hkv) * d].unflatten(1, (hq + hkv, d)), pos, (16, 24, 24), 1.0e6, False, False)
            out, lse = step(qkv, pos, cache, table, ints(start), hq, hkv, d)
            heads = qkv[:, :(hq + hkv) * d].unflatten(1, (hq + hkv, d))
            close(heads, turned, bound)
            want.write(table.tolist(), start, [n, n], heads[:, hq:], qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)))
            same_cache(cache, want, f"after {n}")
            start = [start[0] + n, start[1] + n]
            o, l, o_off, l_off = want.attend(table.tolist(), start, [n, n], heads[:, :hq], d ** -0.5)
            close(out, o, o_off)
            close(lse, l, l_off)


@pytest.mark.parametrize("n", [1, 40])
def test_captured_step_follows_its_inputs(n):
    hq, hkv, d = 28, 4, 128
    g = gen(5)
    cache, plain = pool(g, 12, hkv, d), None
    plain = binding.PageCache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone())
    table, start = tables(g, [300, 300], 12), ints([0, 10])
    qkv, pos = normal(g, 2 * n, (hq + 2 * hkv) * d), torch.zeros((3, 2 * n), dtype=torch.int64, device="cuda")
    steps = []
    for i in range(5):
        steps.append((normal(g, 2 * n, (hq + 2 * hkv) * d), torch.randint(0, 900, (3, 2 * n), device="cuda", generator=g)))
    warm = binding.PageCache.empty(12, hkv, d)
    step(qkv.clone(), pos, warm, table, start, hq, hkv, d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(qkv, pos, cache, table, start, hq, hkv, d)
        scores = binding.token_logprobs(out.flatten(1).float(), torch.zeros(2 * n, dtype=torch.int32, device="cuda"), top=3)
    for i, (x, p) in enumerate(steps):
        qkv.copy_(x)
        pos.copy_(p)
        graph.replay()
        o, l = step(x.clone(), p, plain, table, start, hq, hkv, d)
        assert same_bits(out, o) and same_bits(lse, l), f"step {i}"        # (the second stream's first tokens are junk, NaN among them)
        assert torch.equal(cache.k.view(torch.uint8), plain.k.view(torch.uint8)) and torch.equal(cache.v_scale, plain.v_scale)
        again = binding.token_logprobs(o.flatten(1).float(), torch.zeros(2 * n, dtype=torch.int32, device="cuda"), top=3)
        assert all(same_bits(a, b) for a, b in zip(scores, again))
        start += n


def test_lm_score_is_the_heads_logits_scored():
    g = gen(3)
    d, vocab = 256, 512
    cfg = binding.make_config(1, d, 4, 2, 64, 16, 4, 4, 2, use_rmsnorm=1, out_dtype=1, vocab=vocab)
    w = normal(g, 8 * 64, d, std=0.02)
    lm = normal(g, vocab, d, std=0.1)
    batch = binding.StreamBatch(cfg, [w], lm=(lm, None))
    hidden = normal(g, 6, d, dtype=FP32)
    logits, token = batch.lm_head(hidden)
    lp, entropy, rank, best, best_lp = batch.lm_score(hidden, token, top=5)
    assert rank.tolist() == [0] * 6 and torch.equal(best[:, 0], token)
    want = ref.token_logprobs(logits, token, 5)
    close(lp, torch.tensor([w[0] for w in want], dtype=torch.float64), 1e-5)
    assert [r.tolist() for r in best] == [w[3] for w in want]
    batch.close()
