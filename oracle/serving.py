"""Float64 definitions of what lies between the linears of a decoder layer: many requests' adapters beside a projection, head
norms and rotations into a paged cache, attention over it.  Loops where they say most plainly what is meant.

Beside each result stands the sum of the magnitudes that make it up, where a tolerance needs one.
"""
import math

import numpy as np

E4M3_MAX = 448.0


def e4m3_values():
    """The 256 values of the 8-bit format: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    v = np.empty(256, np.float64)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if (c & 127) == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v[c] = -x if c & 128 else x
    return v


def e4m3_nearest(x):
    """Values of the nearest codes (ties to the even mantissa), saturating; NaN stays NaN."""
    pos = e4m3_values()[:127]                             # ascending, codes 0 .. 126
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), E4M3_MAX)
    hi = np.clip(np.searchsorted(pos, np.where(np.isnan(a), 0.0, a)), 1, 126)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), np.nan, np.copysign(pos[code], x))


def linear_adapters(x, pairs, scalings, adapter_of_row, base):
    """y[m] = base[m] + s_a B_a (A_a x[m]); pairs: list of (A, B) float64.  Returns (y, sum of magnitudes)."""
    y = np.asarray(base, np.float64).copy()
    size = np.abs(y)
    for m in range(y.shape[0]):
        a = int(adapter_of_row[m])
        if not 0 <= a < len(pairs):
            continue
        A, B = pairs[a]
        s = 1.0 if scalings is None else float(scalings[a])
        xm = np.asarray(x[m], np.float64)
        y[m] += s * (B @ (A @ xm))
        size[m] += abs(s) * (np.abs(B) @ (np.abs(A) @ np.abs(xm)))
    return y, size


def head(x, weight, eps, cs, rot, interleaved):
    """One head: norm (weight or None), then the pairs of the first `rot` columns turned by cs (rot/2 x (cos, sin))."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x) + eps) * np.asarray(weight, np.float64)
    y = x.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = float(cs[i][0]), float(cs[i][1])
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def cache_append(q, k, v, q_weight, k_weight, rotations, positions, rot, interleaved, eps):
    """(q, k, v) of every row as they are stored, before the rounding: M x heads x dim float64."""
    def turned(t, weight):
        out = np.empty(t.shape, np.float64)
        for m in range(t.shape[0]):
            known = rot == 0 or 0 <= positions[m] < rotations.shape[0]
            cs = rotations[positions[m]] if rot and known else np.full((rot // 2, 2), np.nan)
            for h in range(t.shape[1]):
                out[m, h] = head(t[m, h], weight, eps, cs, rot, interleaved)
        return out
    return turned(q, q_weight), turned(k, k_weight), np.asarray(v, np.float64)


def cache_attention(q, pages_k, pages_v, page_table, lengths, window, scale):
    """q: B x heads x dim; pages: n_pages x kv x page x dim, float64 values.  Returns (out, lse, sum of p |v|,
    largest |v|, largest sum of |scale q k|)."""
    B, heads, dim = q.shape
    n_pages, kv, page, _ = pages_k.shape
    out, size = np.zeros((B, heads, dim)), np.zeros((B, heads, dim))
    lse, most, logit = np.full((B, heads), -np.inf), np.zeros((B, heads)), np.zeros((B, heads))
    for b in range(B):
        n = min(max(int(lengths[b]), 0), page_table.shape[1] * page)
        at = [t for t in range(max(0, n - window) if window else 0, n) if 0 <= page_table[b, t // page] < n_pages]
        if not at:
            continue
        at = np.array(at)
        p, o = page_table[b, at // page], at % page
        for i in range(heads):
            h = i // (heads // kv)
            K, V = pages_k[p, h, o], pages_v[p, h, o]
            s = scale * (K @ q[b, i])
            top = s.max()
            if top == -np.inf:
                continue
            w = np.exp(s - top)
            out[b, i] = (w @ V) / w.sum()
            size[b, i] = (w @ np.abs(V)) / w.sum()
            lse[b, i] = top + math.log(w.sum())
            most[b, i] = np.abs(V).max()
            logit[b, i] = (abs(scale) * (np.abs(K) @ np.abs(q[b, i]))).max()
    return out, lse, size, most, logit


# ---------------------------------------------------------------------------------------------------- scales by block
BLOCK = 16
LEAST_POWER, MOST_POWER = -15, 8


def block_power(values):
    """The least e of -15 .. 8 with |x| <= 448 2^e for all finite values (-15 where there is none; 8 where no e is large enough)."""
    x = np.abs(np.asarray(values, np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    e = LEAST_POWER
    while e < MOST_POWER and top > E4M3_MAX * 2.0 ** e:
        e += 1
    return e


def block_codes(x, e):
    """Values of the nearest codes to x / 2^e: at most 448, or 240 where e is 8."""
    most = 240.0 if e == MOST_POWER else E4M3_MAX
    return e4m3_nearest(np.clip(np.asarray(x, np.float64) / 2.0 ** e, -most, most))


def cache_append_blocks(rows, slots, codes, powers):
    """rows: M x kv x dim, keys (turned) or values, float64; codes: n_pages x kv x page x dim, values of the codes; powers: n_pages x kv x page / 16.
    Changes codes and powers."""
    n_pages, kv, page, _ = codes.shape
    mine = {}
    for m, s in enumerate(int(s) for s in slots):
        if 0 <= s < n_pages * page:
            mine.setdefault(s // BLOCK, []).append((s % BLOCK, m))
    for block, got in mine.items():
        p, i = block * BLOCK // page, block * BLOCK % page // BLOCK
        for h in range(kv):
            e = block_power(np.stack([rows[m, h] for _, m in got]))
            old = min(max(int(powers[p, h, i]), LEAST_POWER), MOST_POWER)
            here = codes[p, h, BLOCK * i:BLOCK * i + BLOCK]
            if all(place != 0 for place, _ in got):
                e = max(e, old)
                if e != old:
                    here[:] = block_codes(here * 2.0 ** old, e)
            for place, m in got:
                here[place] = block_codes(rows[m, h], e)
            powers[p, h, i] = e


def cache_attention_rows(q, pages_k, pages_v, page_table, lengths, row_starts, window, sinks, scale):
    """q: M x heads x dim; pages: n_pages x kv x page x dim, float64 values.  row_starts None: one row a request.  Rows of no request are NaN.
    Returns (out, lse, sum of p |v|, largest |v|, largest sum of |scale q k|)."""
    M, heads, dim = q.shape
    n_pages, kv, page, _ = pages_k.shape
    B = page_table.shape[0]
    starts = np.arange(B + 1) if row_starts is None else np.clip(np.asarray(row_starts, np.int64), 0, M)
    out, size = np.full((M, heads, dim), np.nan), np.zeros((M, heads, dim))
    lse, most, logit = np.full((M, heads), np.nan), np.zeros((M, heads)), np.zeros((M, heads))
    for b in range(B):
        n, rows = min(max(int(lengths[b]), 0), page_table.shape[1] * page), int(starts[b + 1] - starts[b])
        t = np.arange(n)
        paged = (page_table[b, t // page] >= 0) & (page_table[b, t // page] < n_pages)
        for r in range(rows):
            m, p = int(starts[b]) + r, n - rows + r
            see = paged & (t <= p)
            if window:
                see &= (t > p - window) | (t < sinks)
            at = t[see]
            out[m], lse[m] = 0.0, -np.inf
            if not len(at):
                continue
            pages, place = page_table[b, at // page], at % page
            for h in range(kv):
                mine = slice(h * (heads // kv), (h + 1) * (heads // kv))         # the query heads of this kv head
                K, V = pages_k[pages, h, place], pages_v[pages, h, place]
                with np.errstate(invalid="ignore"):
                    s = scale * (q[m, mine] @ K.T)
                    top = s.max(-1)
                    some = ~(top == -np.inf)
                    w = np.exp(s - np.where(some, top, 0.0)[:, None])
                    total = np.where(some, w.sum(-1), 1.0)
                    if np.isfinite(V).all():
                        o = w @ V
                    else:
                        o = np.stack([np.where(x[:, None] == 0, 0.0, x[:, None] * V).sum(0) for x in w])
                    out[m, mine] = np.where(some[:, None], o / total[:, None], 0.0)
                    size[m, mine] = np.where(some[:, None], (w @ np.abs(V)) / total[:, None], 0.0)
                    lse[m, mine] = np.where(some, top + np.log(total), -np.inf)
                    most[m, mine] = np.abs(V).max()
                    logit[m, mine] = (abs(scale) * (np.abs(q[m, mine]) @ np.abs(K).T)).max(-1)
    return out, lse, size, most, logit
