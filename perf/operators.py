"""The stand-alone operators of this package as measured cases: what a program calls that keeps frames in detail.

The bank keeps one carrier a frame.  A program that also keeps some frames (or all of them) with every visual token does so in a
paged cache of 8-bit keys and values: it rotates the projected rows by their positions (time, height, width), writes them into
the cache, reads them back where another program wants them, and attends over the cache with an answer's token, a question or
whole frames.  What the language-model head says is then scored: the log probability of given answer tokens, as multiple-choice
benchmarks of video models do, with the entropy and the best alternatives.

Two backbones, as in the cases beside this file: the Qwen2-7B shape and a small one with 64-wide heads.  A page of the cache is
64 tokens; key and value codes (e4m3) of a page and head share one scale, a power of two.
"""
import math
import random

import torch

own = False          # True: the package's kernels; False: the same operators in elementary torch operations

BACKBONES = {
    "qwen2_7b": dict(hq=28, hkv=4, hd=128, vocab=152064, sections=(16, 24, 24)),
    "small": dict(hq=16, hkv=4, hd=64, vocab=32000, sections=(8, 12, 12)),
}
PAGE = 64
E_MIN, E_MAX = -110, 120          # exponents a page's scale can have
THETA = 1.0e6


def _rope(name, **kw):
    return dict(dict(name=name, op="rope", backbone="qwen2_7b", rows=1, dtype="bf16", interleaved=False, inverse=False, far=False), **kw)


def _cache(name, op, **kw):
    return dict(dict(name=name, op=op, backbone="qwen2_7b", seqs=1, rows_lo=1, rows_hi=1, held_lo=0, held_hi=0, dtype="bf16",
                     causal=True, window=0, lens=1), **kw)


def _score(name, **kw):
    return dict(dict(name=name, op="score", rows=1, vocab=BACKBONES["qwen2_7b"]["vocab"], top=20, dtype="fp32"), **kw)


def listed():
    return [
        # one answer token's query and key heads, rotated where the projection left them: all latency
        _rope("rope_token"),
        # a clip of 16 frames of 210 tokens and their carriers
        _rope("rope_clip", rows=3376),
        # sixteen viewers' answer tokens, each appended to a cache of its own, mostly into pages that hold tokens already
        _cache("write_tokens", "write", seqs=16, held_lo=700, held_hi=4200, lens=2),
        # a frame of 64 to 256 tokens of each of sixteen streams
        _cache("write_frames", "write", seqs=16, rows_lo=65, rows_hi=257, held_lo=0, held_hi=900, lens=3),
        # a few short stretches of the small backbone's cache, odd lengths, as fp32
        _cache("read_small", "read", backbone="small", seqs=5, rows_lo=33, rows_hi=171, held_lo=0, held_hi=117, dtype="fp32", lens=4),
        # 64 frames of 210 tokens of one stream, for a program that wants them as bf16
        _cache("read_frames", "read", rows_lo=13440, rows_hi=13440),
        # an answer token over 64 frames of 210 tokens
        _cache("attend_token", "attend", held_lo=13503, held_hi=13503),
        # answer tokens of sixteen viewers side by side, two thousand to 64 thousand tokens kept of each
        _cache("attend_tokens", "attend", seqs=16, held_lo=2000, held_hi=65000, lens=5),
        # a question of 32 tokens over 64 frames
        _cache("attend_question", "attend", rows_lo=32, rows_hi=32, held_lo=13440, held_hi=13440),
        # frames of four streams, the cache they stand in long and of different lengths
        _cache("attend_frames", "attend", seqs=4, rows_lo=150, rows_hi=211, held_lo=9000, held_hi=16000, lens=6),
        # an answer token and its twenty best alternatives
        _score("score_token"),
        # four given answers of some fifty tokens
        _score("score_answers", rows=197, top=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 4096 rows to rotate, positions up to 2^31 among them; caches of 1 to 32 sequences with 1 to 4096 rows
    each, 0 to 65536 tokens held; all keys, causal or a window of them; 1 to 256 rows of 1000 to 200000 logits."""
    top = _cost(listed()[9])
    while True:
        op = rng.choice(["rope", "write", "read", "attend", "attend", "attend", "score"])
        backbone = "qwen2_7b" if rng.random() < 0.7 else "small"
        if op == "rope":
            c = _rope("", backbone=backbone, rows=_log_int(rng, 1, 4096), dtype=rng.choice(["bf16", "fp32"]),
                      interleaved=rng.random() < 0.5, inverse=rng.random() < 0.3, far=rng.random() < 0.2)
        elif op == "score":
            c = _score("", rows=_log_int(rng, 1, 256), top=rng.randint(0, 32), dtype=rng.choice(["fp32", "fp32", "bf16"]),
                       vocab=rng.choice([152064, 32000, _log_int(rng, 1000, 200000)]))
        else:
            seqs = _log_int(rng, 1, 32)
            hi = _log_int(rng, 1, 4096 if op != "attend" else 400) if rng.random() < 0.7 else 1
            held = _log_int(rng, 1, 65536 if op == "attend" else 4096)
            c = _cache("", op, backbone=backbone, seqs=seqs, rows_lo=rng.randint(1, hi), rows_hi=hi, held_lo=rng.randint(0, held),
                       held_hi=held, lens=rng.randint(1, 1 << 20))
            if op == "attend":
                c["causal"] = rng.random() < 0.8
                c["window"] = _log_int(rng, 64, 4096) if c["causal"] and rng.random() < 0.2 else 0
            else:
                c["dtype"] = rng.choice(["bf16", "bf16", "fp32"])
        c.pop("name")
        if _cost(c) <= top and _fits(c):
            return c


# ---- sizes ------------------------------------------------------------------------------------------------------------
def _lens(c):
    """(rows, tokens held before them) of each sequence: the case's own, whatever the seed."""
    r = random.Random(c["lens"])
    return [(r.randint(c["rows_lo"], c["rows_hi"]), r.randint(c["held_lo"], c["held_hi"])) for _ in range(c["seqs"])]


def _keys(c, n, held):
    """Keys that the n rows behind `held` tokens see: the pairs, and the keys that any of them sees."""
    total = held + n
    if not c["causal"]:
        return n * total, total
    if not c["window"]:
        return n * held + n * (n + 1) // 2, total
    w = c["window"]
    return sum(min(w, held + t + 1) for t in range(n)), min(total, w + n - 1)


def work(case):
    c = case
    if c["op"] == "score":
        el = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": c["rows"] * (c["vocab"] * el + 16 + 8 * c["top"]), "flops": 5 * c["rows"] * c["vocab"]}
    b = BACKBONES[c["backbone"]]
    el = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "rope":
        n = c["rows"] * (b["hq"] + b["hkv"]) * b["hd"]
        return {"bytes": 2 * n * el + c["rows"] * 24, "flops": 3 * n}
    lens, row = _lens(c), 2 * b["hkv"] * b["hd"]
    rows = sum(n for n, _ in lens)
    pages = sum((n + PAGE - 1) // PAGE for n, _ in lens)
    if c["op"] in ("write", "read"):
        return {"bytes": rows * row * (el + 1) + pages * 8 * b["hkv"], "flops": 2 * rows * row}
    pairs = [_keys(c, n, held) for n, held in lens]
    return {"bytes": 4 * rows * b["hq"] * b["hd"] + 4 * rows * b["hq"] + sum(k for _, k in pairs) * row,
            "flops": 4 * b["hq"] * b["hd"] * sum(p for p, _ in pairs)}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.4e15)


def _fits(c):
    if c["op"] != "attend":
        return True
    b, lens = BACKBONES[c["backbone"]], _lens(c)
    rows, keys = max(n for n, _ in lens), max(n + held for n, held in lens)
    # the plain form lays all sequences out at the longest one's length
    return c["seqs"] * keys * (rows * b["hq"] + 6 * b["hkv"] * b["hd"]) * 4 < 20e9


# ---- inputs -----------------------------------------------------------------------------------------------------------
class _State:
    pass


def _torch_type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def prepare(case, seed):
    c, s = case, _State()
    s.case = dict(c)
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0.0, std, generator=g)

    dtype = _torch_type(c["dtype"])
    if c["op"] == "score":
        # a head's logits: most of the mass on a few tokens; the given tokens are what the model might have said
        s.logits = normal(c["rows"], c["vocab"], std=2.5, dtype=dtype)
        s.tokens = torch.randint(0, c["vocab"], (c["rows"],), device=dev, generator=g, dtype=torch.int32)
        likely = s.logits.argmax(-1).to(torch.int32)
        s.tokens = torch.where(torch.rand(c["rows"], device=dev, generator=g) < 0.7, likely, s.tokens)
        s.outs = None
        return s
    b = BACKBONES[c["backbone"]]
    hq, hkv, hd = b["hq"], b["hkv"], b["hd"]
    e_out = (hq + 2 * hkv) * hd
    if c["op"] == "rope":
        s.qkv = normal(c["rows"], e_out, std=1.2, dtype=dtype)          # a projection's rows: queries, keys, values
        s.x = s.qkv[:, : (hq + hkv) * hd].unflatten(1, (hq + hkv, hd))
        i = torch.arange(c["rows"], device=dev)
        first = int(torch.randint(0, (1 << 31) - 8192 if c["far"] else 30000, (1,), device=dev, generator=g))
        s.positions = torch.stack([first + i // 210, i % 210 // 15, i % 15])     # frames of 14 x 15 patches
        s.sections, s.out = b["sections"], torch.empty((c["rows"], hq + hkv, hd), dtype=dtype, device=dev)
        return s
    lens = _lens(c)
    s.n_rows, s.max_rows = sum(n for n, _ in lens), max(n for n, _ in lens)
    s.uniform = all(n == lens[0][0] for n, _ in lens)
    need = [(n + held + PAGE - 1) // PAGE for n, held in lens]
    n_pages = sum(need) + 3                                              # some pages belong to nobody
    order = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32)
    s.table = torch.full((c["seqs"], max(need) + 1), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(need):
        s.table[i, :n] = order[at:at + n]
        at += n
    s.held = torch.tensor([held for _, held in lens], dtype=torch.int32, device=dev)
    s.offsets = torch.tensor([0] + [n for n, _ in lens], dtype=torch.int32, device=dev).cumsum(0, dtype=torch.int32)
    s.lengths = s.held + s.offsets.diff()
    s.max_len = max(n + held for n, held in lens)

    def pool():
        # pages of normal rows whose size differs by some powers of two: scores of a few units
        e = torch.randint(-7, -4, (n_pages, hkv), device=dev, generator=g)
        codes = torch.empty((n_pages, hkv, PAGE, hd), dtype=torch.float8_e4m3fn, device=dev)
        step = max(1, (1 << 26) // (hkv * PAGE * hd))
        for p in range(0, n_pages, step):
            q = min(step, n_pages - p)
            x = torch.empty((q, hkv, PAGE, hd), device=dev).normal_(0.0, 64.0, generator=g)
            codes[p:p + q] = x.clamp_(-448, 448).to(torch.float8_e4m3fn)
        return codes, torch.exp2(e.float())

    s.k, s.k_scale = pool()
    s.v, s.v_scale = pool()
    s.cache = None
    if c["op"] == "attend":
        s.qkv = normal(s.n_rows, hq * hd, std=1.2)
        s.q = s.qkv.unflatten(1, (hq, hd))
        s.out = torch.empty((s.n_rows, hq, hd), dtype=torch.bfloat16, device=dev)
        s.lse = torch.empty((s.n_rows, hq), device=dev)
    elif c["op"] == "write":
        s.qkv = normal(s.n_rows, e_out, std=1.2, dtype=dtype)
        s.qkv[::97] *= 8                                                 # now and then a row that raises its page's scale
        s.rows_k = s.qkv[:, hq * hd:(hq + hkv) * hd].unflatten(1, (hkv, hd))
        s.rows_v = s.qkv[:, (hq + hkv) * hd:].unflatten(1, (hkv, hd))
    else:
        s.rows_k = torch.empty((s.n_rows, hkv, hd), dtype=dtype, device=dev)
        s.rows_v = torch.empty((s.n_rows, hkv, hd), dtype=dtype, device=dev)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(s):
    op = s.case["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


def _own_rope(s):
    from paper_2503_09387_b200 import binding
    return binding.rope_axes(s.x, s.positions, s.sections, theta=THETA, interleaved=s.case["interleaved"], inverse=s.case["inverse"], out=s.out)


def _own_cache(s):
    if s.cache is None:
        from paper_2503_09387_b200 import binding
        s.cache = binding.PageCache(s.k, s.v, s.k_scale, s.v_scale)
    return s.cache


def _own_write(s):
    _own_cache(s).write(s.table, s.held, s.rows_k, s.rows_v, row_offsets=None if s.uniform else s.offsets)
    return s.k, s.v, s.k_scale, s.v_scale


def _own_read(s):
    return _own_cache(s).read(s.table, s.held, s.rows_k, s.rows_v, row_offsets=None if s.uniform else s.offsets)


def _own_attend(s):
    return _own_cache(s).attend(s.table, s.lengths, s.q, out=s.out, lse=s.lse, row_offsets=None if s.uniform else s.offsets,
                                causal=s.case["causal"], window=s.case["window"])


def _own_score(s):
    from paper_2503_09387_b200 import binding
    s.outs = binding.token_logprobs(s.logits, s.tokens, top=s.case["top"], out=s.outs)
    return s.outs


def _axis_of_pair(sections, interleaved):
    """The axis whose position turns pair k: the sections one behind the other, or the pairs dealt to the axes in turn, an axis
    that has its share left out."""
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    return [a for _, a in sorted((i, a) for a, n in enumerate(sections) for i in range(n))]


def _plain_rope(s):
    half = s.x.shape[-1] // 2
    axis = torch.tensor(_axis_of_pair(s.sections, s.case["interleaved"]), device=s.x.device)
    angle = s.positions[axis].double().T * THETA ** (-torch.arange(half, device=s.x.device).double() / half)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    sin = -sin if s.case["inverse"] else sin
    x = s.x.float()
    lo, hi = x[..., :half], x[..., half:]
    return s.out.copy_(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))


def _places(s):
    """(sequence, place in it, page, row of the page) of each row of the call."""
    r = torch.arange(s.n_rows, device=s.table.device)
    seq = torch.searchsorted(s.offsets, r, right=True) - 1
    t = r - s.offsets[seq]
    pos = (s.held[seq] + t).long()
    return seq, t, s.table[seq, pos // PAGE].long(), pos % PAGE


def _append(s, codes, scale, rows, page, slot):
    x = rows.float()
    amax = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
    opened = torch.zeros(scale.shape[0], dtype=torch.int32, device=x.device).index_add_(0, page, (slot == 0).int()) > 0
    m, e = torch.frexp(amax)                                             # amax = m 2^e, 1/2 <= m < 1;  448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875), E_MIN).clamp(E_MIN, E_MAX)
    e_old = torch.frexp(scale)[1] - 1
    e = torch.where(opened[:, None], e, torch.maximum(e, e_old))
    touched = torch.zeros_like(opened).index_fill_(0, page, True)[:, None]
    # tokens that the page of a sequence's first row holds already
    first = s.table.gather(1, (s.held // PAGE).long()[:, None])[:, 0].long()
    old = codes.view(torch.uint8)[first]
    before = (torch.arange(PAGE, device=x.device) < (s.held % PAGE)[:, None])[:, None, :, None]
    again = torch.ldexp(old.view(torch.float8_e4m3fn).float(), (e_old - e)[first][:, :, None, None]).to(torch.float8_e4m3fn)
    codes.view(torch.uint8)[first] = torch.where(before, again.view(torch.uint8), old)
    q = torch.ldexp(x, -e[page][:, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    codes.view(torch.uint8)[page, :, slot] = q.view(torch.uint8)
    scale.copy_(torch.where(touched, torch.ldexp(torch.ones_like(scale), e), scale))


def _plain_write(s):
    _, _, page, slot = _places(s)
    _append(s, s.k, s.k_scale, s.rows_k, page, slot)
    _append(s, s.v, s.v_scale, s.rows_v, page, slot)
    return s.k, s.v, s.k_scale, s.v_scale


def _values(codes, scale, page, slot):
    return codes.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float() * scale[page][..., None]


def _plain_read(s):
    _, _, page, slot = _places(s)
    return s.rows_k.copy_(_values(s.k, s.k_scale, page, slot)), s.rows_v.copy_(_values(s.v, s.v_scale, page, slot))


def _plain_attend(s):
    c, dev = s.case, s.table.device
    S, L, T = c["seqs"], s.max_len, s.max_rows
    hkv, hd = s.k.shape[1], s.k.shape[3]
    group = s.q.shape[1] // hkv
    pos = torch.arange(L, device=dev)
    page = s.table[:, pos // PAGE].clamp(min=0).long()                   # [S, L]; keys behind a sequence's end are masked below
    slot = (pos % PAGE).expand(S, L)
    k, v = _values(s.k, s.k_scale, page, slot), _values(s.v, s.v_scale, page, slot)
    t = torch.arange(T, device=dev)
    q = s.q[(s.offsets[:-1, None] + t).clamp(max=s.n_rows - 1)].float()
    q = q.unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4)              # [S, Hkv, G, T, D]
    scores = torch.matmul(q.reshape(S, hkv, group * T, hd), k.permute(0, 2, 3, 1)) / math.sqrt(hd)
    at = (s.lengths - s.offsets.diff())[:, None] + t                     # position of row t
    seen = (pos < s.lengths[:, None])[:, None, :].expand(S, T, L)
    if c["causal"]:
        seen = seen & (pos <= at[:, :, None])
    if c["window"]:
        seen = seen & (pos > at[:, :, None] - c["window"])
    scores = scores.view(S, hkv, group, T, L).masked_fill_(~seen[:, None, None], -math.inf)
    m = scores.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = scores.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(S, hkv, group * T, L), v.permute(0, 2, 1, 3)).view(S, hkv, group, T, hd) / total.clamp(min=1e-38)
    lse = (m + total.log())[..., 0]
    seq, i, _, _ = _places(s)
    s.out.copy_(o.permute(0, 3, 1, 2, 4)[seq, i].flatten(1, 2))
    s.lse.copy_(lse.permute(0, 3, 1, 2)[seq, i].flatten(1, 2))
    return s.out, s.lse


def _plain_score(s):
    x = s.logits.float()
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    total = e.sum(-1, keepdim=True)
    lse = (m + total.log())[:, 0]
    given = x.gather(1, s.tokens[:, None].long())
    entropy = total.log()[:, 0] - (e * (x - m)).sum(-1) / total[:, 0]
    index = torch.arange(x.shape[1], device=x.device)
    before = (x > given) | ((x == given) & (index < s.tokens[:, None]))
    bits = (x + 0.0).view(torch.int32)
    ordered = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()      # ascending with x
    key = torch.topk(ordered * (1 << 32) + ((1 << 31) - 1 - index), s.case["top"], dim=-1)[0]
    best = ((1 << 31) - 1 - (key & 0xFFFFFFFF)).to(torch.int32)
    return given[:, 0] - lse, entropy, before.sum(-1).to(torch.int32), best, x.gather(1, best.long()) - lse[:, None]


_OWN = {"rope": _own_rope, "write": _own_write, "read": _own_read, "attend": _own_attend, "score": _own_score}
_PLAIN = {"rope": _plain_rope, "write": _plain_write, "read": _plain_read, "attend": _plain_attend, "score": _plain_score}


# ---- the definitions, in 64 bits --------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "write": _exact_write, "read": _exact_read, "attend": _exact_attend, "score": _exact_score}[case["op"]](s)


def _exact_rope(s):
    # the pair (x_k, x_{k + D/2}) as a complex number, times e^{+-i t}
    half = s.x.shape[-1] // 2
    x = torch.complex(s.x[..., :half].double(), s.x[..., half:].double())
    left, axis = list(s.sections), []
    while any(left):
        if not s.case["interleaved"]:
            axis.append(next(a for a, n in enumerate(left) if n))
            left[axis[-1]] -= 1
            continue
        for a in range(len(left)):
            if left[a]:
                axis.append(a)
                left[a] -= 1
    out = torch.empty_like(x)
    for k, a in enumerate(axis):
        t = s.positions[a].double() * math.exp(-k / half * math.log(THETA))
        out[..., k] = x[..., k] * torch.polar(torch.ones_like(t), -t if s.case["inverse"] else t)[:, None]
    return torch.cat([out.real, out.imag], -1)


def _e4m3(y):
    """The nearest value of the 8-bit format, ties to the even one: a step of 2^-3 of the power of two below, 2^-9 at least."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exact_write(s):
    k, v, ks, vs = s.k.double(), s.v.double(), s.k_scale.double(), s.v_scale.double()
    offsets, held, table = s.offsets.tolist(), s.held.tolist(), s.table.tolist()
    for i in range(len(held)):
        at, end, first = held[i], held[i] + offsets[i + 1] - offsets[i], held[i]
        while at < end:
            page, lo = table[i][at // PAGE], at % PAGE
            n = min(PAGE - lo, end - at)
            r = offsets[i] + at - first
            for codes, scale, rows in ((k, ks, s.rows_k), (v, vs, s.rows_v)):
                x = rows[r:r + n].double().transpose(0, 1)                # [Hkv, n, D]
                amax = x.abs().amax((1, 2)).clamp(min=2.0 ** -200)
                e = torch.ceil(torch.log2(amax / 448))
                e = torch.where(amax > 448 * torch.exp2(e), e + 1, torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e))
                new = torch.exp2(e.clamp(E_MIN, E_MAX))
                if lo:
                    new = torch.maximum(new, scale[page])
                    codes[page][:, :lo] = _e4m3(codes[page][:, :lo] * (scale[page] / new)[:, None, None])
                codes[page][:, lo:lo + n] = _e4m3(x / new[:, None, None])
                scale[page] = new
            at += n
    return k, v, ks, vs


def _gathered(s, codes, scale, i, first, end):
    pages = s.table[i, first // PAGE:(end + PAGE - 1) // PAGE].long()
    x = codes[pages].double() * scale[pages].double()[:, :, None, None]                # [pages, Hkv, 64, D]
    return x.transpose(1, 2).flatten(0, 1)[first % PAGE:first % PAGE + end - first]     # [tokens, Hkv, D]


def _exact_read(s):
    offsets, held = s.offsets.tolist(), s.held.tolist()
    both = [torch.cat([_gathered(s, codes, scale, i, h, h + offsets[i + 1] - offsets[i]) for i, h in enumerate(held)])
            for codes, scale in ((s.k, s.k_scale), (s.v, s.v_scale))]
    return tuple(both)


def _exact_attend(s):
    c = s.case
    offsets, held = s.offsets.tolist(), s.held.tolist()
    hkv, hd = s.k.shape[1], s.k.shape[3]
    group = s.q.shape[1] // hkv
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=s.q.device)
    lse = torch.full(s.q.shape[:2], -math.inf, dtype=torch.float64, device=s.q.device)
    for i, h in enumerate(held):
        lo, hi = offsets[i], offsets[i + 1]
        n, total = hi - lo, h + hi - lo
        k, v = _gathered(s, s.k, s.k_scale, i, 0, total), _gathered(s, s.v, s.v_scale, i, 0, total)
        row, key = torch.arange(h, total, device=k.device)[:, None], torch.arange(total, device=k.device)[None]
        hidden = (key > row) if c["causal"] else torch.zeros((n, total), dtype=torch.bool, device=k.device)
        if c["window"]:
            hidden = hidden | (key <= row - c["window"])
        for head in range(group * hkv):
            scores = s.q[lo:hi, head].double() @ k[:, head // group].T / hd ** 0.5
            scores[hidden] = -math.inf
            lse[lo:hi, head] = torch.logsumexp(scores, -1)
            out[lo:hi, head] = torch.softmax(scores, -1) @ v[:, head // group]
    return out, lse


def _exact_score(s):
    top = s.case["top"]
    lp, entropy, rank, best, best_lp = [], [], [], [], []
    for row, t in zip(s.logits, s.tokens.tolist()):
        x = row.double()
        order = torch.sort(x, descending=True, stable=True)[1]
        logp = torch.log_softmax(x, -1)
        lp.append(logp[t])
        entropy.append(-(logp.exp() * logp).sum())
        rank.append((order == t).nonzero()[0, 0])
        best.append(order[:top])
        best_lp.append(logp[order[:top]])
    return torch.stack(lp), torch.stack(entropy), torch.stack(rank).to(torch.int32), torch.stack(best).to(torch.int32), torch.stack(best_lp)
