"""eora_linear_adapters where rows are put in the order of their pairs: one batch of rows and several, pools whose indices take one and several
passes of the ordering, rows in every order, rows without a pair.

Tolerance, element by element (u = 2^-11: fp16's unit roundoff): u |y| + 2^-16 (sum of magnitudes) + 2^-25: one rounding of y; fp32 sums in chains of at most
some 200 additions, 2^-24 each.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


def draw_ids(kind, M, n, rng):
    if kind == "random":
        return rng.integers(-1, n, M)
    if kind == "one":
        return np.full(M, n - 1)
    if kind == "none but one":
        ids = np.full(M, -1)
        ids[M // 2] = 0
        return ids
    if kind == "none":
        return np.where(np.arange(M) % 2, -7, n)
    if kind == "falling":
        return np.arange(M)[::-1] * n // M
    if kind == "runs of 65":
        return (np.arange(M) // 65 * 7) % n
    assert kind == "in turn"
    return np.arange(M) % n


@pytest.mark.parametrize("M,n,kind", [
    (512, 1, "one"), (512, 3, "random"), (513, 5, "in turn"), (600, 2, "none but one"), (700, 4, "none"), (2047, 63, "falling"), (2048, 64, "random"), (2049, 7, "runs of 65"),
    (2200, 300, "in turn"), (4100, 2, "random"), (5000, 150, "falling"),
])
@pytest.mark.parametrize("bits", [16, 4])
def test_rows_in_order(gpu, M, n, kind, bits):
    import torch

    import synth
    rng = np.random.default_rng(M + n + bits)
    d_in, d_out, r = 256, 304, 64
    pairs, stored = [], []
    for _ in range(n):
        A, B = (rng.normal(0, d_in ** -0.5, (r, d_in))).astype(np.float16), (rng.normal(0, r ** -0.5, (d_out, r))).astype(np.float16)
        if bits == 16:
            stored.append((gpu.pack_factor_f16(A), gpu.pack_factor_f16(B)))
        else:
            (ca, sa), (cb, sb) = synth.quantize_sym4(A, 128), synth.quantize_sym4(B, 64)
            (qa, xa), (qb, xb) = gpu.pack_factor_q4(ca, sa), gpu.pack_factor_q4(cb, sb)
            stored.append((qa, qb, xa, xb))
            A = (ca.astype(np.float64) - 8) * np.repeat(sa.astype(np.float64), 128, 1)
            B = (cb.astype(np.float64) - 8) * np.repeat(sb.astype(np.float64), 64, 1)
        pairs.append((A.astype(np.float64), B.astype(np.float64)))
    pools = [torch.from_numpy(np.concatenate([s[i] for s in stored]).view(np.uint8)).cuda() for i in range(len(stored[0]))] + [None] * (4 - len(stored[0]))
    ids = draw_ids(kind, M, n, rng).astype(np.int32)
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    want, size = base.astype(np.float64), np.abs(base.astype(np.float64))
    for a in range(n):
        rows = ids == a
        t, u = x[rows].astype(np.float64) @ pairs[a][0].T, np.abs(x[rows].astype(np.float64)) @ np.abs(pairs[a][0]).T
        want[rows] += t @ pairs[a][1].T
        size[rows] += u @ np.abs(pairs[a][1]).T
    dx, dids = torch.from_numpy(x).cuda(), torch.from_numpy(ids).cuda()
    ws = gpu.new_adapters_workspace(M, d_in, d_out, r)
    results = []
    for in_place in (False, True, False):
        dbase = torch.from_numpy(base).cuda()
        y = dbase if in_place else torch.full((M, d_out), float("nan"), dtype=torch.float16, device="cuda")
        gpu.linear_adapters(dx, pools[0], pools[1], pools[2], pools[3], None, None, dids, dbase, y, M, d_in, d_out, r, n, bits, ws)
        torch.cuda.synchronize()
        results.append(y.cpu().numpy())
    got = results[0].astype(np.float64)
    tol = 2.0 ** -11 * np.abs(want) + 2.0 ** -16 * size + 2.0 ** -25
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%d of %d off, first at %s" % (bad.sum(), bad.size, tuple(np.argwhere(bad)[0]))
    without = (ids < 0) | (ids >= n)
    assert np.array_equal(results[0][without].view(np.uint16), base[without].view(np.uint16))
    assert all(np.array_equal(results[0].view(np.uint16), t.view(np.uint16)) for t in results[1:]), "in place, or a second time, other bits"


def small_pool(gpu, rng, n, d_in, d_out, r):
    import torch
    pairs = [((rng.normal(0, d_in ** -0.5, (r, d_in))).astype(np.float16), (rng.normal(0, r ** -0.5, (d_out, r))).astype(np.float16)) for _ in range(n)]
    pools = [torch.from_numpy(np.concatenate([gpu.pack_factor_f16(p[i]) for p in pairs])).cuda() for i in range(2)]
    return [(A.astype(np.float64), B.astype(np.float64)) for A, B in pairs], pools


def check(got, x, base, ids, pairs, scalings):
    want, size = base.astype(np.float64), np.abs(base.astype(np.float64))
    for a, (A, B) in enumerate(pairs):
        rows = ids == a
        want[rows] += scalings[a] * (x[rows].astype(np.float64) @ A.T @ B.T)
        size[rows] += abs(scalings[a]) * (np.abs(x[rows].astype(np.float64)) @ np.abs(A).T @ np.abs(B).T)
    bad = ~(np.abs(got.astype(np.float64) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -16 * size + 2.0 ** -25)
    assert not bad.any(), "%d of %d off, first at %s" % (bad.sum(), bad.size, tuple(np.argwhere(bad)[0]))


def test_more_rows_than_a_launch(gpu):
    """65536 + 70 rows: 32 batches in order, then two windows."""
    import torch
    rng = np.random.default_rng(9)
    M, n, d_in, d_out, r = 65536 + 70, 5, 128, 48, 32
    pairs, pools = small_pool(gpu, rng, n, d_in, d_out, r)
    scalings = np.array([1.0, -0.5, 2.0, 0.0, 3.0], np.float32)
    ids = rng.integers(-1, n, M).astype(np.int32)
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    dev = [torch.from_numpy(t).cuda() for t in (x, base, ids, scalings)]
    gpu.linear_adapters(dev[0], pools[0], pools[1], None, None, None, dev[3], dev[2], dev[1], dev[1], M, d_in, d_out, r, n, 16, gpu.new_adapters_workspace(M, d_in, d_out, r))
    torch.cuda.synchronize()
    check(dev[1].cpu().numpy(), x, base, ids, pairs, scalings)


def test_order_changes_between_replays_of_a_graph(gpu):
    """The rows' pairs are read when the graph runs: other indices, other order, the eager bits each time; small calls between use the same workspace."""
    import torch
    rng = np.random.default_rng(10)
    M, n, d_in, d_out, r = 900, 70, 256, 80, 64
    pairs, pools = small_pool(gpu, rng, n, d_in, d_out, r)
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    dx, dbase, ids = torch.from_numpy(x).cuda(), torch.from_numpy(base).cuda(), torch.zeros(M, dtype=torch.int32, device="cuda")
    y, ws = torch.empty_like(dbase), gpu.new_adapters_workspace(M, d_in, d_out, r)

    def step(rows):
        gpu.linear_adapters(dx, pools[0], pools[1], None, None, None, None, ids, dbase, y, rows, d_in, d_out, r, n, 16, ws)

    step(M)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(M)
    for draw in ("random", "in turn", "falling", "none", "random"):
        host = draw_ids(draw, M, n, rng).astype(np.int32)
        ids.copy_(torch.from_numpy(host))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.cpu().numpy()
        check(got, x, base, host, pairs, np.ones(n))
        for rows in (64, 100, M):
            y.zero_()
            step(rows)
            torch.cuda.synchronize()
        assert np.array_equal(got.view(np.uint16), y.cpu().numpy().view(np.uint16))
