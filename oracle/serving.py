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
