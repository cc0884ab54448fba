"""The stand-alone operators from their definitions in 64 bits, on the CPU, one small step at a time; and how far a kernel may be off."""
import math

import torch

PAGE = 64
E_MIN, E_MAX = -110, 120
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def axes_of_pairs(sections, interleaved):
    left, out = list(sections), []
    while sum(left):
        for a in range(len(left)):
            while left[a]:
                out.append(a)
                left[a] -= 1
                if interleaved:
                    break
    return out


def rope(x, positions, sections, theta, interleaved, inverse):
    """-> (y, bound on |error| of fp32 arithmetic before the final rounding)."""
    x = x.double().cpu()
    half = x.shape[-1] // 2
    axes = axes_of_pairs(sections, interleaved)
    y = torch.empty_like(x)
    bound = torch.empty_like(x)
    for k in range(half):
        t = positions[axes[k]].cpu().double() * theta ** (-k / half) * (-1 if inverse else 1)
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        y[..., k] = x[..., k] * c - x[..., k + half] * s
        y[..., k + half] = x[..., k + half] * c + x[..., k] * s
        # a fraction of a turn rounded to fp32 (2^-25 of a turn at most), its sine and cosine to 2 units, two products and a sum; the angle
        # itself in fp64, here and there (2^-50 of the angle)
        off = 2 * math.pi * 2.0 ** -25 + 2 * 2.0 ** -23 + 3 * 2.0 ** -24 + 2.0 ** -50 * t.abs()[:, None]
        bound[..., k] = bound[..., k + half] = (x[..., k].abs() + x[..., k + half].abs()) * off
    return y, bound


def nearest_code(y):
    """The nearest e4m3 value, ties to even, magnitudes above 448 to 448."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6, max=2.0 ** 100)))
    step = torch.exp2(e - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


class Cache:
    """Values of the codes and scales of a paged cache, as fp64 on the CPU."""

    def __init__(self, k, v, k_scale, v_scale):
        self.codes = [t.cpu().float().double() for t in (k, v)]
        self.scale = [t.cpu().double() for t in (k_scale, v_scale)]

    def pages(self, table, i, t):
        page = int(table[i][t // PAGE]) if t // PAGE < len(table[i]) else -1
        return page if 0 <= page < self.codes[0].shape[0] else -1

    def write(self, table, start, lens, k, v):
        for which, rows in enumerate((k, v)):
            rows = rows.cpu().double()
            r = 0
            for i, n in enumerate(lens):
                t, end = start[i], start[i] + n
                while t < end:
                    m = min(PAGE - t % PAGE, end - t)
                    page = self.pages(table, i, t)
                    if page >= 0:
                        self._write(which, page, t % PAGE, rows[r:r + m])
                    t += m
                    r += m

    def _write(self, which, page, at, rows):
        codes, scale = self.codes[which], self.scale[which]
        for h in range(rows.shape[1]):
            x = rows[:, h]
            fine = x[torch.isfinite(x)].abs()
            amax = float(fine.max()) if fine.numel() else 0.0
            e = E_MIN
            while e < E_MAX and amax > 448 * 2.0 ** e:
                e += 1
            if at:
                old = float(scale[page, h])
                e_old = min(max(math.frexp(old)[1] - 1 if old > 0 else E_MIN, E_MIN), E_MAX)
                if e > e_old:
                    codes[page, h, :at] = nearest_code(codes[page, h, :at] * 2.0 ** (e_old - e))
                e = max(e, e_old)
            codes[page, h, at:at + len(x)] = nearest_code(x * 2.0 ** -e)
            scale[page, h] = 2.0 ** e

    def rows(self, which, table, i, t0, t1):
        """[t1 - t0, Hkv, D] values, and which of the tokens there are."""
        hkv, _, d = self.codes[0].shape[1:]
        out, there = torch.zeros((t1 - t0, hkv, d), dtype=torch.float64), torch.zeros(t1 - t0, dtype=torch.bool)
        for t in range(t0, t1):
            page = self.pages(table, i, t)
            if page >= 0:
                out[t - t0] = self.codes[which][page, :, t % PAGE] * self.scale[which][page][:, None]
                there[t - t0] = True
        return out, there

    def attend(self, table, lengths, lens, q, scale, causal=True, window=0):
        """-> (out, lse, bound on |error| of the rows before their rounding, bound of lse)."""
        q = q.cpu().double()
        hkv, d = self.codes[0].shape[1], self.codes[0].shape[3]
        group = q.shape[1] // hkv
        out, off = torch.zeros_like(q), torch.zeros_like(q)
        lse, lse_off = torch.full(q.shape[:2], -math.inf, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
        r = 0
        for i, n in enumerate(lens):
            total = max(int(lengths[i]), 0)
            k, there = self.rows(0, table, i, 0, total)
            v, _ = self.rows(1, table, i, 0, total)
            for t in range(n):
                pos = total - n + t
                j = torch.arange(total)
                seen = there.clone()
                if causal:
                    seen &= j <= pos
                if window:
                    seen &= j > pos - window
                for h in range(q.shape[1]):
                    if not bool(seen.any()):
                        continue
                    kk, vv = k[seen, h // group], v[seen, h // group]
                    s = kk @ q[r, h] * scale
                    p = torch.softmax(s, 0)
                    out[r, h] = p @ vv
                    lse[r, h] = torch.logsumexp(s, 0)
                    # scores: d products summed in fp32, a factor of two roundings, the running maximum's and the exponent's few; weights
                    # to 11 bits and 2^x to 2 units; sums of all keys
                    size = float((kk.abs() @ q[r, h].abs()).max()) * scale
                    ds = (d + 4) * 2.0 ** -24 * size + 6 * 2.0 ** -24 * (float(s.abs().max()) + 256)
                    dw = 2 * ds + 2.0 ** -11 + (len(s) + 64) * 2.0 ** -24
                    off[r, h] = 2 * dw * (p @ vv.abs()) + 2.0 ** -38 * vv.abs().amax(0) * len(s)
                    lse_off[r, h] = dw - 2.0 ** -11 + 2.0 ** -22 * abs(float(lse[r, h]))
                r += 1
        return out, lse, off, lse_off


def token_logprobs(logits, tokens, top):
    """Lists by row: (logprob, entropy, rank, [index], [logprob of it])."""
    got = []
    for row, t in zip(logits.cpu().double(), tokens.cpu().tolist()):
        x = row.tolist()
        key = lambda i: (x[i] != x[i], -x[i] if x[i] == x[i] else 0.0, i)
        order = sorted(range(len(x)), key=key)
        bad = any(v != v or v == math.inf for v in x)
        empty = all(v == -math.inf for v in x)
        if bad or empty:
            lp = lambda i: math.nan if bad else -math.inf
            entropy = math.nan if bad else 0.0
        else:
            m = max(x)
            rest = math.fsum(math.exp(v - m) for v in x) - 1.0 if len(x) > 1 else 0.0
            over = math.log1p(rest)                       # (log sum exp less m: m may be so large that the sum loses this)
            lp = lambda i: (x[i] - m) - over
            entropy = math.fsum(-math.exp(v - m - over) * (v - m - over) for v in x if v > -math.inf)
        got.append((0.0 if t < 0 else (math.nan if t >= len(x) else lp(t)), entropy, order.index(t) if 0 <= t < len(x) else -1,
                    order[:top], [lp(i) for i in order[:top]]))
    return got


def attend_at_once(cache, table, lengths, lens, q, scale, causal=True, window=0, chunk=512):
    """Cache.attend of a PageCache by matrix products in 64 bits where its tensors lie, for calls of many rows.  Every token of a
    sequence has a page.  -> (out, lse, bound on |error| of the rows before their rounding, bound of lse), with |k| |q| in the
    place of |k| . |q|, which it is never below."""
    hkv, d, group = cache.n_kv_heads, cache.head_dim, q.shape[1] // cache.n_kv_heads
    out, off = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    lse_off = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    first = 0
    for i, n in enumerate(lens):
        total = lengths[i]
        pages = table[i, :(total + PAGE - 1) // PAGE].long()
        # [Hkv, tokens, D]
        k, v = ((codes[pages].double() * s[pages].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :total]
                for codes, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        key = torch.arange(total, device=q.device)
        for r in range(0, n, chunk):
            m = min(chunk, n - r)
            pos = (total - n + torch.arange(r, r + m, device=q.device)).repeat(group)[:, None]
            seen = (key <= pos) if causal else torch.ones((m * group, total), dtype=torch.bool, device=q.device)
            if window:
                seen = seen & (key > pos - window)
            some = seen.any(-1)
            for h in range(hkv):
                rows, heads = slice(first + r, first + r + m), slice(h * group, (h + 1) * group)
                x = q[rows, heads].double().transpose(0, 1).flatten(0, 1)                    # [group rows, D]
                s = (x @ k[h].T * scale).masked_fill(~seen, -math.inf)
                p = torch.softmax(s, -1).nan_to_num(0.0)
                hidden = ~seen.any(0)                                                        # (may hold anything)
                vh = v[h].masked_fill(hidden[:, None], 0.0)
                size = k[h].masked_fill(hidden[:, None], 0.0).norm(dim=-1).max() * x.norm(dim=-1) * scale if total else torch.zeros_like(x[:, 0])
                ds = (d + 4) * 2.0 ** -24 * size + 6 * 2.0 ** -24 * (size + 256)
                dw = 2 * ds + 2.0 ** -11 + (seen.sum(-1) + 64) * 2.0 ** -24
                far = 2.0 ** -38 * vh.abs().amax(0) * seen.sum(-1)[:, None] if total else 0.0
                back = lambda t: t.unflatten(0, (group, m)).transpose(0, 1)
                out[rows, heads] = back(p @ vh)
                off[rows, heads] = back(2 * dw[:, None] * (p @ vh.abs()) + far)
                l = torch.logsumexp(s, -1)
                lse[rows, heads] = back(l)
                lse_off[rows, heads] = back(torch.where(some, dw - 2.0 ** -11 + 2.0 ** -22 * l.abs(), 0.0))
        first += n
    return out, lse, off, lse_off
