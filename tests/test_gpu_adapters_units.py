"""eora_linear_adapters where a workgroup has several units of work, one after the other: more pairs and ranks than there are workgroups for, in one launch (up to 64
rows) and by windows (up to 511).

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


def drawn(gpu, rng, n, d_in, d_out, r):
    import torch
    pairs = [((rng.normal(0, d_in ** -0.5, (r, d_in))).astype(np.float16), (rng.normal(0, r ** -0.5, (d_out, r))).astype(np.float16)) for _ in range(n)]
    pool = [torch.from_numpy(np.concatenate([gpu.pack_factor_f16(p[i]) for p in pairs])).cuda() for i in range(2)]
    return [(A.astype(np.float64), B.astype(np.float64)) for A, B in pairs], pool


def check(got, x, base, ids, pairs, ranks):
    want, size = base.astype(np.float64), np.abs(base.astype(np.float64))
    for a, (A, B) in enumerate(pairs):
        rows, k = ids == a, ranks[a]
        want[rows] += x[rows].astype(np.float64) @ A[:k].T @ B[:, :k].T
        size[rows] += np.abs(x[rows].astype(np.float64)) @ np.abs(A[:k]).T @ np.abs(B[:, :k]).T
    bad = ~(np.abs(got.astype(np.float64) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -16 * size + 2.0 ** -25)
    assert not bad.any(), "%d of %d off, first at %s" % (bad.sum(), bad.size, tuple(np.argwhere(bad)[0]))


@pytest.mark.parametrize("M,n,d_in,d_out,r,mixed", [
    (64, 64, 512, 48, 512, False),           # one launch, 512 units of the first part on 256 workgroups
    (64, 64, 512, 48, 512, True),
    (61, 61, 256, 656, 480, True),
    (511, 64, 256, 80, 32, False),           # eight windows of 64 pairs, 32 workgroups each
    (511, 80, 256, 80, 512, False),
    (450, 64, 512, 208, 512, True),
    (333, 97, 128, 48, 160, True),
    (302, 1, 384, 112, 256, False),
])
def test_several_units_a_workgroup(gpu, M, n, d_in, d_out, r, mixed):
    import torch
    rng = np.random.default_rng(M + n + r)
    pairs, pool = drawn(gpu, rng, n, d_in, d_out, r)
    ranks = [32 * int(rng.integers(0, r // 32 + 1)) for _ in range(n)] if mixed else [r] * n
    ids = (np.arange(M) % n).astype(np.int32)
    ids[M // 3] = -1
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    dev = [torch.from_numpy(t).cuda() for t in (x, base, ids, np.array(ranks, np.int32))]
    ws = gpu.new_adapters_workspace(M, d_in, d_out, r)
    first = None
    for _ in range(3):
        y = torch.full((M, d_out), float("nan"), dtype=torch.float16, device="cuda")
        gpu.linear_adapters(dev[0], pool[0], pool[1], None, None, dev[3], None, dev[2], dev[1], y, M, d_in, d_out, r, n, 16, ws)
        torch.cuda.synchronize()
        got = y.cpu().numpy()
        first = got if first is None else first
        assert np.array_equal(got.view(np.uint16), first.view(np.uint16)), "other bits a second time"
    assert gpu.workspace_error(ws) == 0
    check(first, x, base, ids, pairs, ranks)


def test_calls_of_other_sizes_between_replays(gpu):
    """A graph of 900 rows; between its replays calls of 64 and 100 rows on the same workspace, each against the definition."""
    import torch
    rng = np.random.default_rng(11)
    M, n, d_in, d_out, r = 900, 70, 256, 80, 64
    pairs, pool = drawn(gpu, rng, n, d_in, d_out, r)
    x, base = rng.normal(0, 1, (M, d_in)).astype(np.float16), rng.normal(0, 1, (M, d_out)).astype(np.float16)
    dx, dbase, ids = torch.from_numpy(x).cuda(), torch.from_numpy(base).cuda(), torch.zeros(M, dtype=torch.int32, device="cuda")
    y, ws = torch.empty_like(dbase), gpu.new_adapters_workspace(M, d_in, d_out, r)

    def step(rows):
        gpu.linear_adapters(dx, pool[0], pool[1], None, None, None, None, ids, dbase, y, rows, d_in, d_out, r, n, 16, ws)

    step(M)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(M)
    for draw in range(3):
        host = rng.integers(-1, n, M).astype(np.int32)
        ids.copy_(torch.from_numpy(host))
        for rows in (M, 64, 100):
            y.fill_(7.0)
            g.replay() if rows == M else step(rows)
            torch.cuda.synchronize()
            got = y.cpu().numpy()
            check(got[:rows], x[:rows], base[:rows], host[:rows], pairs, [r] * n)
            assert np.all(got[rows:] == 7.0)
    assert gpu.workspace_error(ws) == 0
