"""eora_linear_adapters with NaN and infinities in the pool: where nothing is used, and where it is.  In all three forms: up to 64 rows, to 511, and more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


def call(eora, x, pool, ranks, ids, base, d_in, d_out, r, n, bits):
    import torch
    M = x.shape[0]
    dev = lambda t: None if t is None else torch.from_numpy(np.ascontiguousarray(t.view(np.int32) if t.dtype == np.uint32 else t)).cuda()      # noqa: E731
    y = torch.zeros((M, d_out), dtype=torch.float16, device="cuda")
    eora.linear_adapters(dev(x), *[dev(t) for t in pool], dev(np.array(ranks, np.int32)), None, dev(ids.astype(np.int32)), dev(base), y, M, d_in, d_out, r, n, bits,
                         eora.new_adapters_workspace(M, d_in, d_out, r))
    torch.cuda.synchronize()
    return y.cpu().numpy()


@pytest.mark.parametrize("M", [1, 5, 64, 100, 600])
@pytest.mark.parametrize("bits,r", [(16, 96), (16, 512), (4, 256), (4, 512), (3, 256), (3, 384)])
def test_behind_a_pairs_rank_anything_may_lie(gpu, bits, r, M):
    """Pairs of smaller ranks with NaN in all that is stored behind them (A, B, scales) give, bit for bit, what they give with zeros there."""
    import synth
    rng = np.random.default_rng(M + r + bits)
    d_in, d_out, n, step = 512, 208, 4, 32 if bits == 16 else 128
    ranks = [step, r - step, 0, r]
    pools = [[], []]                         # zeros behind the ranks, NaN
    for k in ranks:
        A, B = rng.normal(0, d_in ** -0.5, (r, d_in)).astype(np.float16), rng.normal(0, r ** -0.5, (d_out, r)).astype(np.float16)
        for pool, fill in zip(pools, (0.0, np.nan)):
            a, b = A.copy(), B.copy()
            if bits == 16:
                a[k:], b[:, k:] = fill, fill
                pool.append((gpu.pack_factor_f16(a), gpu.pack_factor_f16(b)))
            else:
                quant, pack = (synth.quantize_sym4, gpu.pack_factor_q4) if bits == 4 else (synth.quantize_sym3, gpu.pack_factor_q3)
                (ca, sa), (cb, sb) = quant(a, 128), quant(b, 128)
                sa, sb = sa.copy(), sb.copy()
                sa[k:], sb[:, k // 128:] = fill, fill
                (qa, xa), (qb, xb) = pack(ca, sa), pack(cb, sb)
                pool.append((qa, qb, xa, xb))
    pools = [[np.stack([s[i] for s in pool]) for i in range(len(pool[0]))] + [None] * (4 - len(pool[0])) for pool in pools]
    assert any(np.isnan(t.view(np.float16)).any() for t in pools[1] if t is not None)
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    ids = rng.integers(-1, n, M)
    ids[0] = 0
    clean, got = (call(gpu, x, p, ranks, ids, base, d_in, d_out, r, n, bits) for p in pools)
    assert np.isfinite(clean.astype(np.float64)).all()
    assert np.array_equal(got.view(np.uint16), clean.view(np.uint16)), "%d values changed" % (got.view(np.uint16) != clean.view(np.uint16)).sum()


@pytest.mark.parametrize("M", [1, 5, 64, 100, 600])
@pytest.mark.parametrize("r,ranks", [(64, [64, 32, 64]), (512, [32, 512, 480])])
def test_infinities_in_b(gpu, r, ranks, M):
    """An infinite element of B makes y infinite, with the sign of t's element, and NaN where that is zero; the other outputs are what they are without it."""
    rng = np.random.default_rng(M + r)
    d_in, d_out, n = 256, 80, 3
    A = [rng.normal(0, d_in ** -0.5, (r, d_in)).astype(np.float16) for _ in range(n)]
    B = [rng.normal(0, r ** -0.5, (d_out, r)).astype(np.float16) for _ in range(n)]
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    ids = rng.integers(-1, n, M)
    ids[0] = 0
    if M > 2:
        ids[2], x[2] = 1, 0                  # t = 0
    pool = lambda: [np.stack([gpu.pack_factor_f16(t) for t in m]) for m in (A, B)] + [None, None]      # noqa: E731
    clean = call(gpu, x, pool(), ranks, ids, base, d_in, d_out, r, n, 16)
    # (output, rank, sign) of the infinities in each pair
    at = [[(3, 7, 1), (17, 31, -1)], [(0, 0, -1), (40, ranks[1] - 1, 1)], [(79, 5, 1)]]
    for b, some in zip(B, at):
        for o, c, sign in some:
            b[o, c] = sign * np.inf
    want = clean.astype(np.float64)
    for m in range(M):
        if ids[m] < 0:
            continue
        t = A[ids[m]].astype(np.float64) @ x[m].astype(np.float64)
        for o, c, sign in at[ids[m]]:
            want[m, o] = sign * np.inf * t[c] if t[c] else np.nan
    got = call(gpu, x, pool(), ranks, ids, base, d_in, d_out, r, n, 16).astype(np.float64)
    assert np.array_equal(got, want, equal_nan=True), "%d values off" % (~((got == want) | (np.isnan(got) & np.isnan(want)))).sum()
