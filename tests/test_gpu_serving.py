"""GPU parity of eora_linear_adapters, eora_cache_append and eora_cache_attention against the float64 definitions of
oracle/serving.py, at the sizes, masks and values where they can go wrong.

Tolerances, element by element (u = 2^-11: fp16's unit roundoff):
  adapters   u |y| + 2^-16 (sum of magnitudes) + 2^-25: one rounding of y; fp32 sums in chains of at most some 200 additions, 2^-24 each
  append     u |y| + 2^-20 (largest value of the head) + 2^-25: one rounding; a dozen fp32 operations.  8 bits: as near as the nearest
             code, but for 2^-18 (largest value of the head, in code units)
  attention  1.25 u (|out| + sum p |v|) + tokens 2^-24 max|v| + 2^-25: a weight and the result are rounded to fp16 once each, and weights below
             2^-14 of the reference lose bits; lse: 2^-17 (1 + largest sum |scale q k|): fp32 dot products
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -11
TINY = 2.0 ** -25


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


def close(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), what + ": NaN in other places"
    with np.errstate(invalid="ignore"):
        bad = ~nan & ~(got == want) & ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, first at %s: %r for %r, allowed %r" % (
        what, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), got[bad][0], want[bad][0], np.broadcast_to(tol, want.shape)[bad][0])


# ---------------------------------------------------------------------------------------------------- adapters
class Pool:
    """n pairs of rank up to r, some smaller (zeros behind), stored with the library's packers; their values in float64."""

    def __init__(self, eora, seed, d_in, d_out, r, n, bits, ranks=None, size=1.0):
        import torch

        import synth
        from oracle import linear
        rng = np.random.default_rng(seed)
        self.pairs, stored = [], []
        for a in range(n):
            A = (rng.normal(0, size * d_in ** -0.5, (r, d_in))).astype(np.float16)
            B = (rng.normal(0, r ** -0.5, (d_out, r))).astype(np.float16)
            if bits == 16:
                stored.append((eora.pack_factor_f16(A), eora.pack_factor_f16(B), None, None))
            else:
                quant, pack = (synth.quantize_sym4, eora.pack_factor_q4) if bits == 4 else (synth.quantize_sym3, eora.pack_factor_q3)
                wide = min(128, r)
                (ca, sa), (cb, sb) = quant(A, 128), quant(B, wide)
                (qa, xa), (qb, xb) = pack(ca, sa), pack(cb, sb)
                stored.append((qa, qb, xa, xb))
                zero = 1 << (bits - 1)
                A = linear.dequant(ca, np.full(sa.shape, zero), sa, 128)
                B = linear.dequant(cb, np.full(sb.shape, zero), sb, wide)
            k = r if ranks is None else max(0, min(r, ranks[a]))
            self.pairs.append((A[:k].astype(np.float64), B[:, :k].astype(np.float64)))
        put = lambda i: None if stored[0][i] is None else torch.from_numpy(      # noqa: E731
            np.stack([s[i].view(np.int32) if s[i].dtype == np.uint32 else s[i] for s in stored])).cuda()
        self.A, self.B, self.As, self.Bs = (put(i) for i in range(4))
        self.args = (d_in, d_out, r, n, bits)
        self.ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device="cuda")


def run_adapters(eora, pool, x, ids, scalings, base, in_place=False, ws=None):
    """y (M x d_out fp16 numpy), with a canary on both sides of it."""
    import torch
    d_in, d_out, r, n, bits = pool.args
    M, pad = x.shape[0], 64
    buf = torch.full((M * d_out + 2 * pad,), 777.0, dtype=torch.float16, device="cuda")
    y = buf[pad:pad + M * d_out].view(M, d_out)
    b = None
    if base is not None:
        b = torch.from_numpy(base).cuda()
        if in_place:
            y.copy_(b)
            b = y
    ws = eora.new_adapters_workspace(M, d_in, d_out, r) if ws is None else ws
    s = None if scalings is None else torch.tensor(scalings, dtype=torch.float32, device="cuda")
    eora.linear_adapters(torch.from_numpy(x).cuda(), pool.A, pool.B, pool.As, pool.Bs, pool.ranks, s, torch.tensor(ids, dtype=torch.int32, device="cuda"), b, y,
                         M, d_in, d_out, r, n, bits, ws)
    torch.cuda.synchronize()
    out = buf.cpu().numpy()
    assert np.all(out[:pad] == 777.0) and np.all(out[pad + M * d_out:] == 777.0), "write outside y"
    return out[pad:pad + M * d_out].reshape(M, d_out)


def check_adapters(eora, pool, x, ids, scalings, base, **kw):
    from oracle import serving
    y = run_adapters(eora, pool, x, ids, scalings, base, **kw)
    want, size = serving.linear_adapters(x, pool.pairs, scalings, ids, np.zeros(y.shape) if base is None else base)
    close(y, want, U * np.abs(want) + 2.0 ** -16 * size + TINY, "adapters")
    return y


ADAPTERS = [
    # M, d_in, d_out, r, n, bits, mixed ranks
    (1, 128, 16, 32, 1, 16, False),
    (1, 1024, 1024, 64, 4, 16, True),
    (2, 512, 48, 96, 3, 16, True),
    (17, 640, 272, 128, 5, 16, True),        # seventeen rows: more than one block of one pair
    (64, 256, 64, 32, 1, 16, False),         # a whole window of one pair
    (65, 384, 112, 64, 2, 16, True),         # a second window of one row
    (130, 256, 528, 32, 9, 16, True),
    (600, 128, 144, 32, 3, 16, False),       # ten windows: few leaders each, several rounds of them
    (5, 4096, 64, 512, 2, 16, True),         # the largest rank, LDS beyond 64 KiB with more rows below
    (70, 2048, 80, 512, 2, 16, True),
    (3, 512, 32, 64, 3, 4, False),           # 4-bit pairs of rank 64: B's tiles are 64 wide
    (33, 384, 96, 256, 4, 4, True),
    (9, 256, 48, 128, 3, 3, False),
    (80, 640, 80, 256, 3, 3, True),
]


@pytest.mark.parametrize("M,d_in,d_out,r,n,bits,mixed", ADAPTERS)
def test_adapters_shapes(gpu, M, d_in, d_out, r, n, bits, mixed):
    rng = np.random.default_rng(M * 31 + d_out)
    step = 32 if bits == 16 else min(128, r)
    ranks = [step * int(rng.integers(0, r // step + 1)) for _ in range(n)] if mixed else None
    pool = Pool(gpu, M + r, d_in, d_out, r, n, bits, ranks)
    x = rng.normal(0, 1, (M, d_in)).astype(np.float16)
    base = rng.normal(0, 1, (M, d_out)).astype(np.float16)
    ids = rng.integers(-1, n, M)
    ids[0] = n - 1
    s = rng.uniform(0.5, 2, n).astype(np.float32)
    y = check_adapters(gpu, pool, x, ids, s, base)
    again = run_adapters(gpu, pool, x, ids, s, base, in_place=True)
    assert np.array_equal(y.view(np.uint16), again.view(np.uint16)), "in place, or a second time, other bits"
    check_adapters(gpu, pool, x, ids, None, None)


@pytest.mark.parametrize("bits,r", [(16, 96), (16, 256), (16, 384), (16, 512), (4, 64), (4, 256), (3, 128), (3, 384)])
def test_adapters_many_rows(gpu, bits, r):
    """From 512 rows on, blocks of rows of one pair share its tiles; pairs of few rows and rows without one lie between them."""
    rng = np.random.default_rng(r + bits)
    pool = Pool(gpu, 60 + r, 256, 336, r, 4, bits, [r, r // 2 if bits == 16 else r, r, 0])
    ids = np.concatenate([np.repeat([1, 0, -1, 2, 3], [130, 200, 5, 190, 3]), rng.integers(-1, 4, 30)])
    x, base = rng.normal(0, 1, (len(ids), 256)).astype(np.float16), rng.normal(0, 1, (len(ids), 336)).astype(np.float16)
    step = 32 if bits == 16 else min(128, r)
    for a, k in enumerate([r, r // 2 if bits == 16 else r, r, 0]):       # ranks go up to whole tiles
        up = -(-k // step) * step
        if up != k:
            pool.pairs[a] = tuple(t.astype(np.float64) for t in _first(pool, gpu, 60 + r, 256, 336, r, 4, a, up))
    y = check_adapters(gpu, pool, x, ids, [1.0, -0.5, 2.0, 1.0], base)
    again = run_adapters(gpu, pool, x, ids, [1.0, -0.5, 2.0, 1.0], base, in_place=True)
    assert np.array_equal(y.view(np.uint16), again.view(np.uint16))


def test_adapters_runs_of_prompts(gpu):
    """300 rows of four prompts, one without a pair: runs that begin and end inside windows."""
    rng = np.random.default_rng(5)
    pool = Pool(gpu, 6, 512, 320, 64, 3, 16)
    ids = np.repeat([1, 2, -1, 0], [100, 77, 3, 120])
    check_adapters(gpu, pool, rng.normal(0, 1, (300, 512)).astype(np.float16), ids, [1.0, 0.5, -2.0], rng.normal(0, 1, (300, 320)).astype(np.float16))


def test_adapters_indices_and_ranks_out_of_range(gpu):
    """Rows whose index names no pair, and pairs of no rank, are base bit for bit; ranks above r are r; others go up to whole tiles."""
    rng = np.random.default_rng(7)
    pool = Pool(gpu, 8, 256, 64, 96, 4, 16, [0, 1000, 40, -5])
    pool.pairs[2] = tuple(t.astype(np.float64) for t in _first(pool, gpu, 8, 256, 64, 96, 4, 2, 64))
    x, base = rng.normal(0, 1, (8, 256)).astype(np.float16), rng.normal(0, 1, (8, 64)).astype(np.float16)
    ids = [-1, 4, -2 ** 31, 2 ** 31 - 1, 0, 3, 1, 2]
    y = check_adapters(gpu, pool, x, ids, None, base)
    assert np.array_equal(y[:6].view(np.uint16), base[:6].view(np.uint16))
    assert not run_adapters(gpu, pool, x, ids, None, None)[:6].any()


def _first(pool, eora, seed, d_in, d_out, r, n, a, k):
    """The first k ranks of pair a, drawn as Pool draws them."""
    rng = np.random.default_rng(seed)
    for i in range(a + 1):
        A = rng.normal(0, d_in ** -0.5, (r, d_in)).astype(np.float16)
        B = rng.normal(0, r ** -0.5, (d_out, r)).astype(np.float16)
    return A[:k], B[:, :k]


@pytest.mark.parametrize("bits", [16, 4])
def test_adapters_large_and_small_t(gpu, bits):
    """t far outside fp16's range, either way, and rows of very different size in one block: t is scaled row by row."""
    rng = np.random.default_rng(9)
    pool = Pool(gpu, 10, 512, 64, 128, 1, bits, size=16.0)
    x = rng.normal(0, 1, (20, 512)) * np.array([6e4, 1.0, 1e-3, 1e-6, 0.0] * 4)[:, None]
    x = np.clip(x, -65000, 65000).astype(np.float16)
    base = np.zeros((20, 64), np.float16)
    check_adapters(gpu, pool, x, np.zeros(20, int), [2.0 ** -9], base)
    check_adapters(gpu, pool, x[[1, 2, 3, 4]], np.zeros(4, int), [1024.0], base[:4])


def test_adapters_expired_wait(gpu):
    """With every wait counted as expired the call ends and says so; a workspace zeroed again works as before."""
    import torch
    rng = np.random.default_rng(15)
    pool = Pool(gpu, 16, 512, 256, 64, 3, 16)
    x, base, ids = rng.normal(0, 1, (9, 512)).astype(np.float16), rng.normal(0, 1, (9, 256)).astype(np.float16), rng.integers(-1, 3, 9)
    ws = gpu.new_adapters_workspace(9, 512, 256, 64)
    want = run_adapters(gpu, pool, x, ids, None, base, ws=ws)
    assert gpu.workspace_error(ws) == 0
    gpu.debug_set_spin_limit(-1)
    try:
        run_adapters(gpu, pool, x, ids, None, base, ws=ws)
        assert gpu.workspace_error(ws) == -8
    finally:
        gpu.debug_set_spin_limit(1 << 22)
    ws.zero_()
    for _ in range(3):
        assert np.array_equal(run_adapters(gpu, pool, x, ids, None, base, ws=ws).view(np.uint16), want.view(np.uint16))
    assert gpu.workspace_error(ws) == 0
    assert not ws.view(torch.int32)[:64 + 32 * 64].any()     # the counts are left at zero


def test_adapters_one_workspace_for_calls_of_all_sizes(gpu):
    rng = np.random.default_rng(17)
    pool = Pool(gpu, 18, 384, 272, 128, 5, 16, [128, 0, 32, 96, 64])
    ws = gpu.new_adapters_workspace(600, 384, 272, 128)
    x, base = rng.normal(0, 1, (600, 384)).astype(np.float16), rng.normal(0, 1, (600, 272)).astype(np.float16)
    base[:, 3] = -0.0
    for M in (1, 64, 600, 17, 65, 2, 64):
        ids = rng.integers(-1, 5, M)
        y = check_adapters(gpu, pool, x[:M], ids, None, base[:M], ws=ws)
        none = (ids < 0) | (ids == 1)
        assert np.array_equal(y[none].view(np.uint16), base[:M][none].view(np.uint16))
    assert gpu.workspace_error(ws) == 0


def test_adapters_infinities_stay_in_their_row(gpu):
    rng = np.random.default_rng(11)
    pool = Pool(gpu, 12, 256, 32, 32, 2, 16)
    x, base = rng.normal(0, 1, (6, 256)).astype(np.float16), rng.normal(0, 1, (6, 32)).astype(np.float16)
    ids = np.array([0, 0, 1, 1, 0, -1])
    clean = run_adapters(gpu, pool, x, ids, None, base)
    x[1, 3], x[2, 7], x[5, 0] = np.inf, np.nan, np.nan
    base[4, 5] = -np.inf
    y = run_adapters(gpu, pool, x, ids, None, base).astype(np.float32)
    assert not np.isfinite(y[1]).any() and np.isnan(y[2]).all() and y[4, 5] == -np.inf
    clean[4, 5] = -np.inf
    for m in (0, 3, 4, 5):
        assert np.array_equal(y[m], clean[m].astype(np.float32))


def test_adapters_pool_beyond_32_bits(gpu):
    """A pool of more than 2^32 bytes (and halves): the last slots are found."""
    import torch
    rng = np.random.default_rng(13)
    small = Pool(gpu, 14, 1024, 1024, 512, 2, 16)
    n = 2 ** 32 // (1024 * 512) + 3
    big = Pool.__new__(Pool)
    big.A, big.B = (torch.empty((n, 1024 * 512), dtype=torch.float16, device="cuda") for _ in range(2))
    big.A[n - 2:], big.B[n - 2:] = small.A, small.B
    big.As = big.Bs = big.ranks = None
    big.args = (1024, 1024, 512, n, 16)
    x, base = rng.normal(0, 1, (3, 1024)).astype(np.float16), rng.normal(0, 1, (3, 1024)).astype(np.float16)
    got = run_adapters(gpu, big, x, [n - 1, n - 2, -1], None, base)
    want = run_adapters(gpu, small, x, [1, 0, -1], None, base)
    assert np.array_equal(got.view(np.uint16), want.view(np.uint16))


# ---------------------------------------------------------------------------------------------------- append
def rotations(n, rot):
    f = 10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    a = np.arange(n)[:, None] * f
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def append_case(seed, M, heads, kv, dim, bits, page, norm, rot, pages, stride_pad=0):
    """Numpy inputs; q, k and v are parts of one buffer where stride_pad is given."""
    rng = np.random.default_rng(seed)
    c = dict(M=M, heads=heads, kv=kv, dim=dim, bits=bits, page=page, rot=rot, pages=pages)
    c["q"], c["k"], c["v"] = (rng.normal(0, 1, (M, h, dim)).astype(np.float16) for h in (heads, kv, kv))
    c["qw"] = rng.normal(1, 0.2, dim).astype(np.float16) if norm in ("both", "q") else None
    c["kw"] = rng.normal(1, 0.2, dim).astype(np.float16) if norm in ("both", "k") else None
    c["table"] = rotations(200, rot) if rot else None
    c["positions"] = rng.integers(0, 200, M).astype(np.int32)
    c["slots"] = rng.permutation(pages * page)[:M].astype(np.int64)
    c["ks"], c["vs"] = (rng.uniform(0.005, 0.02, kv).astype(np.float32) if bits == 8 else None for _ in range(2))
    c["pad"] = stride_pad
    return c


def run_append(eora, c, interleaved=False, eps=1e-5, in_place=False):
    """(q_out, k pages, v pages) as float64 values, codes' values for 8 bits; the pages held 7.0 before."""
    import torch
    M, heads, kv, dim, pad = (c[k] for k in ("M", "heads", "kv", "dim", "pad"))
    dev = lambda t: None if t is None else torch.from_numpy(np.ascontiguousarray(t)).cuda()      # noqa: E731
    q, k, v = dev(c["q"]), dev(c["k"]), dev(c["v"])
    strides = (heads * dim, kv * dim, kv * dim)
    if pad:
        row = (heads + 2 * kv) * dim + pad
        buf = torch.full((M, row), 999.0, dtype=torch.float16, device="cuda")
        at = [0, heads * dim, (heads + kv) * dim, (heads + 2 * kv) * dim]
        for t, lo, hi in ((q, at[0], at[1]), (k, at[1], at[2]), (v, at[2], at[3])):
            buf[:, lo:hi] = t.view(M, -1)
        q, k, v = buf[:, at[0]:at[1]], buf[:, at[1]:at[2]], buf[:, at[2]:at[3]]
        strides = (row,) * 3
    guard = 64
    out = torch.full((M * heads * dim + 2 * guard,), 777.0, dtype=torch.float16, device="cuda")
    q_out = q if in_place else out[guard:guard + M * heads * dim]
    kind = torch.float8_e4m3fn if c["bits"] == 8 else torch.float16
    pk, pv = (torch.full((c["pages"], kv, c["page"], dim), 7.0, device="cuda").to(kind) for _ in range(2))
    eora.cache_append(q, k, v, dev(c["qw"]), dev(c["kw"]), dev(c["table"]), dev(c["positions"]), dev(c["slots"]), q_out, pk, pv, dev(c["ks"]), dev(c["vs"]),
                      M, heads, kv, dim, *strides, c["rot"], interleaved, 200 if c["rot"] else 0, eps, c["pages"], c["page"], c["bits"])
    torch.cuda.synchronize()
    full = out.cpu().numpy()
    assert np.all(full[:guard] == 777.0) and np.all(full[guard + M * heads * dim:] == 777.0), "write outside q_out"
    return q_out.float().cpu().numpy().reshape(M, heads, dim), pk.float().cpu().numpy().astype(np.float64), pv.float().cpu().numpy().astype(np.float64)


def check_append(eora, c, interleaved=False, eps=1e-5, **kw):
    from oracle import serving
    q, pk, pv = run_append(eora, c, interleaved, eps, **kw)
    wq, wk, wv = serving.cache_append(c["q"], c["k"], c["v"], c["qw"], c["kw"], c["table"], c["positions"], c["rot"], interleaved, eps)

    def tol(w):
        with np.errstate(invalid="ignore"):
            return U * np.abs(w) + 2.0 ** -20 * np.nanmax(np.abs(w), -1, initial=0.0, keepdims=True) + TINY

    close(q, wq, tol(wq), "q")
    for got, want, scale, name in ((pk, wk, c["ks"], "k"), (pv, wv, c["vs"], "v")):
        untouched = np.ones(got.shape, bool)
        for m in range(c["M"]):
            s = int(c["slots"][m])
            if not 0 <= s < c["pages"] * c["page"]:
                continue
            one = got[s // c["page"], :, s % c["page"]]
            untouched[s // c["page"], :, s % c["page"]] = False
            if c["bits"] == 16:
                close(one, want[m], tol(want[m]), "%s of row %d" % (name, m))
            else:
                x = want[m] / scale[:, None].astype(np.float64)
                near = serving.e4m3_nearest(x)
                clipped = np.clip(x, -448, 448)
                with np.errstate(invalid="ignore"):
                    room = 2.0 ** -18 * np.nanmax(np.abs(clipped), -1, initial=0.0, keepdims=True)
                    bad = ~(np.abs(one - clipped) <= np.abs(near - clipped) + room) & ~np.isnan(x)
                assert not bad.any() and np.array_equal(np.isnan(one), np.isnan(x)), "%s of row %d" % (name, m)
        assert np.all(got[untouched] == 7.0), "%s: a place that no row names was written" % name


APPENDS = [
    # M, heads, kv, dim, bits, page, norm, rot, interleaved, pages
    (1, 32, 8, 128, 16, 16, "", 128, False, 2),
    (1, 1, 1, 64, 16, 16, "both", 64, False, 1),
    (3, 5, 1, 64, 8, 48, "q", 16, True, 2),
    (7, 12, 3, 64, 16, 48, "both", 48, False, 3),         # a third of a head's pairs lies in other lanes' halves
    (5, 7, 7, 128, 8, 16, "k", 96, False, 2),
    (40, 4, 2, 256, 16, 32, "both", 256, True, 3),
    (33, 3, 1, 256, 8, 16, "both", 240, False, 4),
    (70, 2, 2, 128, 16, 64, "both", 0, False, 2),          # norms alone
    (2, 80, 10, 64, 8, 16, "", 0, False, 1),               # neither: q and v as they are
    (1100, 1, 1, 64, 16, 16, "both", 16, False, 70),       # more tokens than workgroups for a slice of heads
]


@pytest.mark.parametrize("M,heads,kv,dim,bits,page,norm,rot,interleaved,pages", APPENDS)
def test_append_shapes(gpu, M, heads, kv, dim, bits, page, norm, rot, interleaved, pages):
    check_append(gpu, append_case(M + heads + dim, M, heads, kv, dim, bits, page, norm, rot, pages), interleaved)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_from_one_buffer_and_in_place(gpu, bits):
    check_append(gpu, append_case(21, 9, 6, 2, 128, bits, 16, "both", 128, 2, stride_pad=24))
    check_append(gpu, append_case(22, 9, 6, 2, 128, bits, 16, "both", 64, 2), in_place=True)


def test_append_padding_rows_and_positions_out_of_range(gpu):
    c = append_case(23, 8, 4, 2, 64, 16, 16, "both", 32, 2)
    c["slots"][[0, 3, 5]] = [-1, 32, -2 ** 62]            # not stored; 32 is one past the last
    c["positions"][[1, 2]] = [-1, 200]                     # their rotated columns are NaN, the others not
    check_append(gpu, c)
    c = append_case(24, 8, 4, 2, 64, 8, 16, "", 32, 2)
    c["positions"][4] = 2 ** 31 - 1
    check_append(gpu, c, True)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_extreme_values(gpu, bits):
    """A zero head (eps alone), values at fp16's ends, 8-bit values beyond 448, NaN: each in its own head only."""
    c = append_case(25, 6, 3, 2, 64, bits, 16, "q", 64, 1)
    c["q"][0, 1] = 0
    c["q"][1, 2] = 6e4
    c["q"][2, 0] *= 2.0 ** -20
    c["k"][3, 0, 5] = np.nan
    c["v"][4, 1, 7] = np.nan
    c["v"][5] *= 1000
    check_append(gpu, c)


# ---------------------------------------------------------------------------------------------------- attention
class Cache:
    """A cache of random values whose unused places hold NaN; requests' pages in any order."""

    def __init__(self, seed, lengths, heads, kv, dim, bits, page, width=None, k_size=1.0, q_size=1.0, q_pad=0):
        import torch
        rng = np.random.default_rng(seed)
        B = len(lengths)
        used = [-(-n // page) for n in lengths]
        width = max([1] + used) if width is None else width
        n_pages = sum(used) + 2
        order = rng.permutation(n_pages)
        self.table = rng.choice(np.array([-1, n_pages, 2 ** 31 - 1, -2 ** 31]), (B, width)).astype(np.int32)
        self.k = np.full((n_pages, kv, page, dim), np.nan)
        self.v = np.full((n_pages, kv, page, dim), np.nan)
        at = 0
        for b, n in enumerate(lengths):
            for p in range(used[b]):
                here = min(page, n - p * page)
                self.table[b, p] = order[at]
                self.k[order[at], :, :here] = rng.normal(0, k_size, (kv, here, dim))
                self.v[order[at], :, :here] = rng.normal(0, 1, (kv, here, dim))
                at += 1
        self.bits, self.page, self.kv, self.dim, self.heads, self.B, self.width, self.n_pages = bits, page, kv, dim, heads, B, width, n_pages
        self.lengths = np.array(lengths, np.int32)
        self.q = rng.normal(0, q_size, (B, heads, dim)).astype(np.float16)
        self.q_pad = q_pad
        self.set(rng)

    def set(self, rng=None):
        """Stored tensors from the values, and the values from what is stored."""
        import torch
        if self.bits == 16:
            self.dk, self.dv = (torch.from_numpy(t.astype(np.float16)).cuda() for t in (self.k, self.v))
            self.ks = self.vs = None
            self.k, self.v = (t.double().cpu().numpy() for t in (self.dk, self.dv))
            return
        self.ks, self.vs = (torch.from_numpy(rng.uniform(0.01, 0.03, self.kv).astype(np.float32)).cuda() for _ in range(2))
        self.dk, self.dv = ((torch.from_numpy(t).cuda() / s[:, None, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn)
                            for t, s in ((self.k, self.ks), (self.v, self.vs)))
        self.k, self.v = ((t.float().double() * s.double()[:, None, None]).cpu().numpy() for t, s in ((self.dk, self.ks), (self.dv, self.vs)))

    def run(self, eora, window=0, scale=None, ws=None, lse=True):
        import torch
        row = self.heads * self.dim + self.q_pad
        q = torch.full((self.B, row), np.nan, dtype=torch.float16, device="cuda")
        q[:, :self.heads * self.dim] = torch.from_numpy(self.q).cuda().view(self.B, -1)
        guard, size = 64, self.B * self.heads * self.dim
        buf = torch.full((size + 2 * guard,), 777.0, dtype=torch.float16, device="cuda")
        out = buf[guard:guard + size]
        got = torch.full((self.B * self.heads + 8,), 777.0, dtype=torch.float32, device="cuda")
        ws = eora.new_attention_workspace(self.B, self.heads, self.kv, self.dim, self.width * self.page) if ws is None else ws
        eora.cache_attention(q, self.dk, self.dv, self.ks, self.vs, torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda(), out,
                             got[4:-4] if lse else None, self.B, self.heads, self.kv, self.dim, row, self.n_pages, self.page, self.bits, self.width, window,
                             self.dim ** -0.5 if scale is None else scale, ws)
        torch.cuda.synchronize()
        full, l = buf.cpu().numpy(), got.cpu().numpy()
        assert np.all(full[:guard] == 777.0) and np.all(full[guard + size:] == 777.0), "write outside out"
        assert np.all(l[:4] == 777.0) and np.all(l[-4:] == 777.0), "write outside lse"
        return full[guard:guard + size].reshape(self.B, self.heads, self.dim), l[4:-4].reshape(self.B, self.heads)

    def check(self, eora, window=0, scale=None, **kw):
        from oracle import serving
        out, lse = self.run(eora, window, scale, **kw)
        want, wl, size, most, logit = serving.cache_attention(self.q.astype(np.float64), self.k, self.v, self.table, self.lengths, window,
                                                              self.dim ** -0.5 if scale is None else scale)
        n = np.maximum(self.lengths, 0)[:, None, None]
        close(out, want, 1.25 * U * (np.abs(want) + size) + n * 2.0 ** -24 * most[..., None] + TINY, "out")
        close(lse, wl, 2.0 ** -17 * (1 + logit), "lse")
        return out, lse


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 200]
ATTENTION = [
    # lengths, heads, kv, dim, bits, page
    ([1], 1, 1, 64, 16, 16),
    ([100], 32, 8, 128, 16, 16),
    (EDGES, 8, 2, 128, 16, 16),
    (EDGES, 8, 2, 128, 8, 16),
    (EDGES, 5, 5, 64, 16, 48),               # one query head each, pages that are no power of two
    (EDGES, 6, 1, 64, 8, 80),
    (EDGES, 4, 1, 256, 16, 32),
    (EDGES, 3, 3, 256, 8, 16),
    ([40, 0, 300], 16, 1, 128, 16, 16),      # a full block of query heads
    ([40, 0, 300], 17, 1, 128, 16, 16),      # and one more
    ([70, 1, 555], 40, 2, 64, 8, 16),        # blocks of 16 and of 4
    ([2049], 16, 1, 256, 16, 256),           # the widest heads and a full block: LDS beyond 64 KiB
    ([5000], 8, 2, 128, 16, 64),             # one request over many workgroups
    ([9000, 3, 0, 1], 4, 1, 128, 8, 16),     # one long, others short
    ([0, 0, 0], 4, 2, 64, 16, 16),           # nothing at all
]


@pytest.mark.parametrize("lengths,heads,kv,dim,bits,page", ATTENTION)
def test_attention_shapes(gpu, lengths, heads, kv, dim, bits, page):
    c = Cache(len(lengths) + heads + dim + bits, lengths, heads, kv, dim, bits, page)
    out, lse = c.check(gpu)
    again = c.run(gpu, lse=False)[0]
    assert np.array_equal(out.view(np.uint16), again.view(np.uint16)), "a second time, or without lse, other bits"


@pytest.mark.parametrize("window", [1, 16, 31, 100, 10 ** 9])
@pytest.mark.parametrize("bits", [16, 8])
def test_attention_window(gpu, window, bits):
    Cache(31, EDGES + [700], 4, 2, 64, bits, 16).check(gpu, window=window)


def test_attention_many_requests(gpu):
    """More requests than a workgroup has threads: their tiles are counted in rounds."""
    rng = np.random.default_rng(32)
    Cache(33, [int(n) for n in rng.integers(0, 40, 600)], 2, 1, 64, 16, 16).check(gpu)


def test_attention_lengths_beyond_the_table_and_missing_pages(gpu):
    c = Cache(34, [90, 64, 33, 50], 4, 2, 64, 16, 16, width=6)
    c.lengths[:] = [90, -7, 33, 50]
    c.table[2, 1] = -1                       # tokens 16 .. 31 of the third request are masked
    c.table[3] = -1                          # the last one has no page at all
    out, lse = c.check(gpu)
    assert not out[1].any() and not out[3].any() and np.all(lse[[1, 3]] == -np.inf)
    c = Cache(35, [96, 64], 4, 2, 64, 8, 16, width=6)
    c.lengths[0] = 2 ** 31 - 1               # as far as the table goes
    c.lengths[1] = 64
    from oracle import serving
    want = serving.cache_attention(c.q.astype(np.float64), c.k, c.v, c.table, [96, 64], 0, 0.125)
    out, lse = c.run(gpu)
    close(out, want[0], 1.25 * U * (np.abs(want[0]) + want[2]) + 1e-5, "out")


def test_attention_rising_scores_and_large_ones(gpu):
    """Scores that rise along the cache raise the reference many times; large ones leave one weight."""
    for bits in (16, 8):
        c = Cache(36, [1500, 777], 4, 1, 128, bits, 16, k_size=1.0)
        for b in range(2):
            for t in range(c.lengths[b]):
                c.k[c.table[b, t // 16], :, t % 16] = c.q[b].mean(0) * (t / 200.0) + 0.1 * c.k[c.table[b, t // 16], :, t % 16]
        c.set(np.random.default_rng(37))
        c.check(gpu, scale=0.5)
    Cache(38, [600, 33], 8, 2, 64, 16, 16, k_size=8.0, q_size=8.0).check(gpu)
    c = Cache(39, [300], 4, 1, 64, 16, 16)
    c.check(gpu, scale=0.0)                  # all weights alike
    c.check(gpu, scale=-0.25)


def test_attention_infinities_and_nan(gpu):
    """A score of -inf masks its token; NaN and +inf scores make NaN of their own heads only."""
    c = Cache(40, [70, 70, 70], 2, 2, 64, 16, 16)
    c.q[0] = np.abs(c.q[0])
    c.k[c.table[0, 1], 0, 3] = -np.inf
    c.k[c.table[1, 2], 1, 5, 7] = np.nan
    c.v[c.table[2, 0], 0, 1, 9] = np.inf
    c.set()
    clean = Cache(40, [70, 70, 70], 2, 2, 64, 16, 16)
    clean.q[0] = np.abs(clean.q[0])
    out, lse = c.check(gpu)
    base, _ = clean.check(gpu)
    assert np.isnan(out[1, 1]).all() and np.array_equal(out[1, 0], base[1, 0]) and np.array_equal(out[2, 1], base[2, 1])
    assert out[2, 0, 9] == np.inf and np.array_equal(np.delete(out[2, 0], 9), np.delete(base[2, 0], 9))


def test_attention_rows_of_a_wider_buffer_and_several_tokens_of_one_request(gpu):
    c = Cache(41, [50, 50, 50], 4, 2, 128, 16, 16, q_pad=72)
    c.table[1:] = c.table[0]
    c.lengths[:] = [48, 49, 50]
    c.check(gpu)


def test_attention_joins_with_lse(gpu):
    """Two halves of a cache, joined by their lse, are the whole."""
    c = Cache(42, [4096], 8, 2, 128, 16, 64)
    out, lse = c.run(gpu)
    whole, table = c.table.copy(), c.table
    parts = []
    for half in (0, 1):
        c.table = np.ascontiguousarray(whole[:, 32 * half:32 * half + 32])
        c.width, c.lengths = 32, np.array([2048], np.int32)
        parts.append(c.run(gpu))
    w = np.exp(np.stack([p[1] for p in parts]).astype(np.float64) - lse)
    assert np.allclose(w.sum(0), 1, atol=1e-5)
    joined = sum(p[0].astype(np.float64) * x[..., None] for p, x in zip(parts, w))
    assert np.abs(joined - out).max() <= 4 * U * np.abs(out.astype(np.float64)).max() + 1e-5


def test_attention_and_append_beyond_32_bits(gpu):
    """Pages behind 2^32 elements of a pool."""
    import torch
    c = Cache(43, [40, 17], 4, 2, 64, 16, 16)
    out, lse = c.run(gpu)
    n = 2 ** 32 // (2 * 16 * 64) + 7
    big = [torch.empty((n, 2, 16, 64), dtype=torch.float16, device="cuda") for _ in range(2)]
    for t, small in zip(big, (c.dk, c.dv)):
        t[n - c.n_pages:] = small
    c.dk, c.dv = big
    c.table = np.where((c.table >= 0) & (c.table < c.n_pages), c.table + n - c.n_pages, -1).astype(np.int32)
    c.n_pages = n
    got = c.run(gpu)
    assert np.array_equal(got[0].view(np.uint16), out.view(np.uint16)) and np.array_equal(got[1], lse)
    q, k, v = (torch.randn((1, h, 64), device="cuda").half() for h in (4, 2, 2))
    slot = torch.tensor([n * 16 - 1], device="cuda")
    gpu.cache_append(q, k, v, None, None, None, None, slot, torch.empty_like(q), *big, None, None, 1, 4, 2, 64, 256, 128, 128, 0, False, 0, 0.0, n, 16, 16)
    torch.cuda.synchronize()
    assert torch.equal(big[0][n - 1, :, 15], k[0]) and torch.equal(big[1][n - 1, :, 15], v[0])


# ---------------------------------------------------------------------------------------------------- together
def test_on_another_stream_and_in_a_graph(gpu):
    """The three calls on a stream of their own, then captured and replayed with work between: the eager bits each time."""
    import torch
    pool = Pool(gpu, 50, 256, 512, 32, 3, 16)
    c = Cache(51, [200, 3, 64], 4, 2, 128, 16, 16)
    dev = lambda t: torch.from_numpy(np.ascontiguousarray(t)).cuda()      # noqa: E731
    rng = np.random.default_rng(52)
    x, ids, table = dev(rng.normal(0, 1, (3, 256)).astype(np.float16)), dev(np.array([2, -1, 0], np.int32)), dev(c.table)
    base, q, kvs = torch.zeros((3, 512), device="cuda").half(), torch.empty((3, 512), device="cuda").half(), dev(rng.normal(0, 1, (3, 256)).astype(np.float16))
    lengths, positions = dev(c.lengths), dev(np.array([199, 2, 63], np.int32))
    slots = dev(np.array([c.table[b, (n - 1) // 16] * 16 + (n - 1) % 16 for b, n in enumerate(c.lengths)], np.int64))
    cs, out = dev(rotations(200, 128)), torch.empty((3, 512), device="cuda").half()
    w1, w2 = gpu.new_adapters_workspace(3, 256, 512, 32), gpu.new_attention_workspace(3, 4, 2, 128, c.width * 16)

    def step():
        gpu.linear_adapters(x, pool.A, pool.B, None, None, None, None, ids, base, q, 3, 256, 512, 32, 3, 16, w1)
        gpu.cache_append(q, kvs, kvs, None, None, cs, positions, slots, q, c.dk, c.dv, None, None, 3, 4, 2, 128, 512, 256, 256, 128, False, 200, 0.0, c.n_pages, 16, 16)
        gpu.cache_attention(q, c.dk, c.dv, None, None, table, lengths, out, None, 3, 4, 2, 128, 512, c.n_pages, 16, 16, c.width, 0, 0.1, w2)

    step()
    torch.cuda.synchronize()
    want, keys = out.clone(), c.dk.clone()
    assert torch.isfinite(want).all()
    out.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        out.zero_()
        q.zero_()
        c.dk.copy_(torch.where(torch.isnan(keys), keys, keys))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        x.mul_(1.0)


@pytest.mark.parametrize("heads,kv,dim,bits,page,window", [(8, 2, 64, 16, 16, 0), (6, 3, 128, 16, 48, 0), (8, 8, 128, 8, 16, 70), (4, 2, 256, 16, 32, 0), (16, 1, 64, 8, 64, 0), (5, 5, 256, 8, 16, 33)])
def test_attention_tables_wider_than_the_requests(gpu, heads, kv, dim, bits, page, window):
    """Tables with room for caches that are read past the last-level cache: 128 MiB and more, of which the requests have little."""
    c = Cache(61 + dim + bits, [700, 0, 1, 333, page, 4 * page + 1], heads, kv, dim, bits, page)
    each = 6 * kv * dim * (bits // 8) * 2
    tokens = -(-2 ** 27 // each) if not window else 0
    more = max(0, -(-tokens // page) - c.width) + 3
    c.table = np.ascontiguousarray(np.pad(c.table, ((0, 0), (0, more)), constant_values=-1))
    c.width += more
    c.check(gpu, window)
