"""GPU parity of eora_cache_append_blocks and eora_cache_read against the float64 definitions of oracle/serving.py.

Values meet no arithmetic before they are stored: their codes and powers are the oracle's, bit for bit.  Queries as in eora_cache_append(): u |q| + 2^-20 (largest value of
the head) + 2^-25 (u = 2^-11: one rounding; a dozen fp32 operations).  Keys go through the same operations: 2^-20 of the head's largest value away from the oracle's, so a
power may differ from the oracle's only where the block's largest key is that near to a border (2^-18 of it asked for), and a code is as near to the key, in code units, as the
nearest code is, but for 2^-18 of the head's largest.
"""
import numpy as np
import pytest

from tests.test_gpu_serving import TINY, U, close, rotations

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


def dev(t):
    import torch
    return None if t is None else torch.from_numpy(np.ascontiguousarray(t)).cuda()


class Store:
    """A cache of random codes and powers, and rows for some of its slots."""

    def __init__(self, seed, slots, heads, kv, dim, page, pages, norm="", rot=0, size=1.0, spread=0):
        rng = np.random.default_rng(seed)
        self.slots = np.array(slots, np.int64)
        M = self.M = len(slots)
        self.heads, self.kv, self.dim, self.page, self.pages, self.rot = heads, kv, dim, page, pages, rot
        grow = 2.0 ** rng.integers(-spread, spread + 1, (M, 1, 1)) if spread else 1.0
        self.q = rng.normal(0, 1, (M, heads, dim)).astype(np.float16)
        self.k = (rng.normal(0, size, (M, kv, dim)) * grow).astype(np.float16)
        self.v = (rng.normal(0, size, (M, kv, dim)) * grow).astype(np.float16)
        weight = lambda: (1 + 0.2 * rng.normal(size=dim)).astype(np.float16)       # noqa: E731
        self.qw, self.kw = weight() if norm in ("q", "both") else None, weight() if norm in ("k", "both") else None
        self.table = rotations(200, rot) if rot else None
        self.positions = rng.integers(0, 200, M).astype(np.int32) if rot else None
        self.codes = [rng.choice(256, (pages, kv, page, dim)).astype(np.uint8) for _ in range(2)]
        for c in self.codes:
            c[(c & 127) == 127] = 0x38
        self.bytes = [rng.integers(112, 136, (pages, kv, page // 16)).astype(np.uint8) for _ in range(2)]

    def run(self, eora, interleaved=False, eps=1e-5, pad=0, in_place=False):
        import torch
        M, heads, kv, dim = self.M, self.heads, self.kv, self.dim
        q, k, v = dev(self.q), dev(self.k), dev(self.v)
        strides = (heads * dim, kv * dim, kv * dim)
        if pad:
            row = (heads + 2 * kv) * dim + pad
            buf = torch.full((M, row), 999.0, dtype=torch.float16, device="cuda")
            at = [0, heads * dim, (heads + kv) * dim, (heads + 2 * kv) * dim]
            for t, lo, hi in zip((q, k, v), at, at[1:]):
                buf[:, lo:hi] = t.view(M, -1)
            q, k, v = (buf[:, lo:hi] for lo, hi in zip(at, at[1:]))
            strides = (row,) * 3
        guard = 64
        out = torch.full((M * heads * dim + 2 * guard,), 777.0, dtype=torch.float16, device="cuda")
        q_out = q if in_place else out[guard:guard + M * heads * dim]
        pages = [dev(c) for c in self.codes]
        scales = [torch.cat((torch.full((5,), 77, dtype=torch.uint8, device="cuda"), dev(b).flatten(), torch.full((5,), 77, dtype=torch.uint8, device="cuda"))) for b in self.bytes]
        eora.cache_append_blocks(q, k, v, dev(self.qw), dev(self.kw), dev(self.table), dev(self.positions), dev(self.slots), q_out, *pages, scales[0][5:-5], scales[1][5:-5],
                                 M, heads, kv, dim, *strides, self.rot, interleaved, 200 if self.rot else 0, eps, self.pages, self.page)
        torch.cuda.synchronize()
        full = out.cpu().numpy()
        assert np.all(full[:guard] == 777.0) and np.all(full[guard + M * heads * dim:] == 777.0), "write outside q_out"
        for s in scales:
            assert torch.all(s[:5] == 77) and torch.all(s[-5:] == 77), "write outside the scales"
        self.dev = pages, [s[5:-5].clone() for s in scales]
        return q_out.float().cpu().numpy().reshape(M, heads, dim), [p.cpu().numpy() for p in pages], [s[5:-5].cpu().numpy().reshape(b.shape) for s, b in zip(scales, self.bytes)]

    def check(self, eora, interleaved=False, eps=1e-5, **kw):
        from oracle import serving
        q, codes, got_bytes = self.run(eora, interleaved, eps, **kw)
        wq, wk, wv = serving.cache_append(self.q, self.k, self.v, self.qw, self.kw, self.table, self.positions, self.rot, interleaved, eps)
        with np.errstate(invalid="ignore"):
            close(q, wq, U * np.abs(wq) + 2.0 ** -20 * np.nanmax(np.abs(wq), -1, initial=0.0, keepdims=True) + TINY, "q")
        value = serving.e4m3_values()
        touched = np.zeros(self.bytes[0].shape, bool)
        for s in self.slots:
            if 0 <= s < self.pages * self.page:
                touched[s // self.page, :, s % self.page // 16] = True
        wide = np.repeat(touched, 16, -1)
        for got, byte, old, old_byte, rows, name in ((codes[1], got_bytes[1], self.codes[1], self.bytes[1], wv, "v"), (codes[0], got_bytes[0], self.codes[0], self.bytes[0], wk, "k")):
            assert np.array_equal(got[~wide], old[~wide]) and np.array_equal(byte[~touched], old_byte[~touched]), name + ": a block that no row names was written"
            want, power = value[old], old_byte.astype(int) - 127
            serving.cache_append_blocks(rows, self.slots, want, power)
            if name == "v":
                assert np.array_equal(byte.astype(int) - 127, power), "powers of v"
                assert np.array_equal(value[got], want, equal_nan=True), "codes of v"
                continue
            self.check_keys(serving, value, got, byte.astype(int) - 127, old, old_byte.astype(int) - 127, rows)
        return codes, got_bytes

    def check_keys(self, serving, value, got, power, old, old_power, rows):
        """Block by block: a power that is right for keys 2^-18 larger or smaller, and the nearest codes at it."""
        where = {}
        for m, s in enumerate(int(s) for s in self.slots):
            if 0 <= s < self.pages * self.page:
                where.setdefault(s // 16, []).append((s % 16, m))
        for block, mine in where.items():
            p, i = block * 16 // self.page, block * 16 % self.page // 16
            begun = any(place == 0 for place, _ in mine)
            for h in range(self.kv):
                x = np.stack([rows[m, h] for _, m in mine])
                was = min(max(int(old_power[p, h, i]), -15), 8)
                right = [serving.block_power(x * f) for f in (1 - 2.0 ** -18, 1 + 2.0 ** -18)]
                right = [e if begun else max(e, was) for e in right]
                e = int(power[p, h, i])
                assert e in right, "power of k: %d for %s" % (e, right)
                here = value[got[p, h, 16 * i:16 * i + 16]]
                most = 240.0 if e == 8 else 448.0
                for place, m in mine:
                    want = np.clip(rows[m, h] / 2.0 ** e, -most, most)
                    near = serving.block_codes(rows[m, h], e)
                    with np.errstate(invalid="ignore"):
                        bad = ~(np.abs(here[place] - want) <= np.abs(near - want) + 2.0 ** -18 * np.nanmax(np.abs(want), initial=0.0)) & ~np.isnan(want)
                    assert not bad.any() and np.array_equal(np.isnan(here[place]), np.isnan(want)), "k of row %d" % m
                others = [place for place in range(16) if place not in [q for q, _ in mine]]
                had = value[old[p, h, 16 * i:16 * i + 16]]
                want = had if begun or e == was else serving.block_codes(had * 2.0 ** was, e)
                assert np.array_equal(here[others], want[others], equal_nan=True), "codes of k that were there"


def run_of(first, n):
    return list(range(first, first + n))


CASES = [
    # slots, heads, kv, dim, page, pages, norm, rot, interleaved
    ([5], 32, 8, 128, 16, 2, "", 128, False),
    ([16], 1, 1, 64, 16, 2, "both", 64, False),
    (run_of(0, 16), 4, 2, 128, 16, 1, "both", 128, True),
    (run_of(7, 33), 5, 1, 64, 48, 2, "q", 16, True),      # ends and begins inside blocks
    (run_of(48, 100), 12, 3, 64, 48, 4, "both", 48, False),
    ([95, 3, 40, 16, 71], 7, 7, 128, 32, 3, "k", 96, False),        # requests with one new token each
    (run_of(3, 20) + run_of(67, 5) + [-1, -1] + run_of(130, 14), 4, 2, 256, 32, 5, "both", 256, True),
    (run_of(32, 70), 3, 1, 256, 16, 8, "both", 240, False),
    (run_of(1, 300), 2, 2, 128, 64, 5, "both", 0, False),
    ([31, 30, 29, 28, 1, 0, 2], 80, 10, 64, 16, 2, "", 0, False),   # backwards
    (run_of(0, 1100), 1, 1, 64, 16, 70, "both", 16, False),
    (run_of(5, 2100), 1, 8, 64, 80, 27, "", 0, False),              # wavefronts with more than one block
    (run_of(5, 4200), 1, 40, 64, 16, 264, "", 0, False),            # sixteen rows a wavefront
]


@pytest.mark.parametrize("slots,heads,kv,dim,page,pages,norm,rot,interleaved", CASES)
def test_shapes(gpu, slots, heads, kv, dim, page, pages, norm, rot, interleaved):
    Store(len(slots) + heads + dim, slots, heads, kv, dim, page, pages, norm, rot, spread=3).check(gpu, interleaved)


def test_from_one_buffer_and_in_place(gpu):
    Store(21, run_of(9, 9), 6, 2, 128, 16, 2, "both", 128).check(gpu, pad=24)
    Store(22, run_of(9, 9), 6, 2, 128, 16, 2, "both", 64).check(gpu, in_place=True)


def test_padding_rows_and_positions_out_of_range(gpu):
    c = Store(23, run_of(3, 20), 4, 2, 64, 16, 2, "both", 32)
    c.slots[[0, 4, 5, 19]] = [-1, 32, -2 ** 62, 2 ** 40]
    c.positions[[1, 2]] = [-1, 200]                       # their rotated columns are NaN: they say nothing of the block's power
    c.check(gpu)


def test_scale_of_every_size(gpu):
    """Blocks of zeros, of fp16's least and largest values, of infinities; powers at both ends; a block that was at any of them before."""
    for size in (0.0, 2.0 ** -24, 2.0 ** -20, 1e-3, 300.0, 2e4):
        Store(24, run_of(0, 16) + run_of(37, 11), 2, 2, 64, 32, 2, size=size).check(gpu)
    c = Store(25, run_of(3, 13) + run_of(16, 16), 2, 2, 64, 32, 1)
    c.v[0], c.v[13, 0], c.v[13, 1] = 65504, 57344, 57376
    c.k[0] = -65504
    c.check(gpu)
    c = Store(26, run_of(0, 4), 2, 2, 64, 16, 1)
    c.v[:, 0], c.v[1, 1, 5], c.v[2, 1, 6], c.v[3, 1, 7] = np.inf, np.nan, -np.inf, 448
    c.check(gpu)
    c = Store(27, [4], 2, 2, 64, 16, 1)
    c.bytes[0][:], c.bytes[1][:] = 0, 255                 # taken as the nearest that there are
    c.check(gpu)


def test_grows_token_by_token(gpu):
    """Sixteen calls into one block, each value twice the last: codes that were there are rounded again each time, as the oracle does it."""
    from oracle import serving
    c = Store(28, [0], 2, 1, 128, 16, 1)
    codes, bytes_ = c.codes, c.bytes
    rng = np.random.default_rng(29)
    for t in range(16):
        c.slots[:] = t
        c.v = (rng.normal(0, 2.0 ** (t - 8), c.v.shape)).astype(np.float16)
        c.k = c.v.copy()
        c.codes, c.bytes = c.check(gpu)
    assert c.bytes[1][0, 0, 0] > 127 - 4


def test_beyond_32_bits_and_two_rows_with_one_slot(gpu):
    import torch
    n = 2 ** 32 // (2 * 64 * 64) + 7                       # pages of 8 KiB: 4 GiB and more
    pages = [torch.zeros((n, 2, 64, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((n, 2, 4), dtype=torch.uint8, device="cuda") for _ in range(2)]
    k = torch.randn((2, 2, 64), device="cuda").half()
    slot = torch.tensor([n * 64 - 1, 17], device="cuda")
    gpu.cache_append_blocks(k, k, k, None, None, None, None, slot, torch.empty_like(k), *pages, *scales, 2, 2, 2, 64, 128, 128, 128, 0, False, 0, 0.0, n, 64)
    back = [torch.empty((3, 2, 64), dtype=torch.float16, device="cuda") for _ in range(2)]
    gpu.cache_read(*pages, *scales, torch.tensor([n * 64 - 1, n * 64, 17], device="cuda"), *back, 3, 2, 64, n, 64, 8, 16)
    torch.cuda.synchronize()
    for b in back:
        assert not b[1].any() and (b[[0, 2]] - k).abs().max() <= k.abs().max() / 16
    # one of the two is stored, with a power that holds both
    two = torch.stack((k[0], 100 * k[1]))
    gpu.cache_append_blocks(two, two, two, None, None, None, None, torch.tensor([3, 3], device="cuda"), torch.empty_like(two), *pages, *scales, 2, 2, 2, 64, 128, 128, 128, 0, False,
                            0, 0.0, n, 64)
    gpu.cache_read(*pages, *scales, torch.tensor([3], device="cuda"), *back, 1, 2, 64, n, 64, 8, 16)
    torch.cuda.synchronize()
    most = two.abs().amax().item()
    assert min((back[1][0].float() - two[i].float()).abs().max().item() for i in range(2)) <= most / 16


@pytest.mark.parametrize("kv,dim,page", [(1, 64, 16), (3, 128, 48), (5, 256, 32)])
@pytest.mark.parametrize("form", ["fp16", "heads", "blocks"])
def test_read(gpu, kv, dim, page, form):
    """fp16 and block scales bit for bit; a scale a head with one rounding."""
    import torch

    from oracle import serving
    rng = np.random.default_rng(kv + dim)
    pages, value = 5, serving.e4m3_values()
    if form == "fp16":
        held = [rng.integers(0, 2 ** 16, (pages, kv, page, dim)).astype(np.uint16).view(np.float16) for _ in range(2)]
        scales, want = [None, None], [h.astype(np.float64) for h in held]
    else:
        held = [rng.integers(0, 256, (pages, kv, page, dim)).astype(np.uint8) for _ in range(2)]
        if form == "heads":
            scales = [rng.uniform(0.001, 200, kv).astype(np.float32) for _ in range(2)]
            want = [value[h] * s.astype(np.float64)[:, None, None] for h, s in zip(held, scales)]
        else:
            scales = [rng.integers(112, 136, (pages, kv, page // 16)).astype(np.uint8) for _ in range(2)]
            want = [value[h] * np.repeat(2.0 ** (s.astype(int) - 127), 16, -1)[..., None] for h, s in zip(held, scales)]
    slots = np.concatenate((rng.integers(0, pages * page, 70), [-1, pages * page, 2 ** 62, -2 ** 63, 0, pages * page - 1]))
    guard = 64
    out = [torch.full((len(slots) * kv * dim + 2 * guard,), 777.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    gpu.cache_read(*(dev(h) for h in held), *(dev(s) for s in scales), dev(slots), *(o[guard:-guard] for o in out), len(slots), kv, dim, pages, page, 16 if form == "fp16" else 8,
                   16 if form == "blocks" else 0)
    torch.cuda.synchronize()
    for o, w in zip(out, want):
        full = o.cpu().numpy()
        assert np.all(full[:guard] == 777.0) and np.all(full[-guard:] == 777.0), "write outside"
        got = full[guard:-guard].reshape(len(slots), kv, dim)
        for m, s in enumerate(slots):
            exact = w[s // page, :, s % page] if 0 <= s < pages * page else np.zeros((kv, dim))
            with np.errstate(over="ignore"):
                assert np.array_equal(got[m], exact.astype(np.float16), equal_nan=True) if form != "heads" else np.all(
                    (np.abs(got[m] - exact) <= U * 1.001 * np.abs(exact) + TINY) | (np.isnan(got[m]) & np.isnan(exact)) | (np.abs(exact) >= 65500)), "row %d" % m


def test_more_rows_than_a_launch_takes(gpu):
    """2^18 rows are a launch: a block whose rows are in two of them, and all behind it, are as a call with the last rows alone stores them."""
    import torch
    M, page, dim = (1 << 18) + 40, 16, 64
    first = (1 << 18) - 9 - 32                               # a row whose slot, 9 further on, begins a block
    pages = (M + 9) // page + 1
    torch.manual_seed(3)
    q, k, v = (torch.randn((M, dim), device="cuda").half() for _ in range(3))
    slots = torch.arange(9, M + 9, device="cuda")
    assert int(slots[first]) % 16 == 0
    results = []
    for m in (0, first):
        cache = [torch.full((pages, 1, page, dim), 0x38, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.full((pages, 1, 1), 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
        out = torch.empty_like(q[m:])
        gpu.cache_append_blocks(q[m:], k[m:], v[m:], None, None, None, None, slots[m:], out, *cache, M - m, 1, 1, dim, dim, dim, dim, 0, False, 0, 0.0, pages, page)
        torch.cuda.synchronize()
        begin = int(slots[first]) // page
        results.append([out[first - m:]] + [c[begin:] for c in cache])
        if m == 0:                                           # and all of the first rows came there: codes of values whose largest is 448 2^e at most, 224 2^e at least
            got = [torch.empty((M, 1, dim), dtype=torch.float16, device="cuda") for _ in range(2)]
            gpu.cache_read(*cache, slots, *got, M, 1, dim, pages, page, 8, 16)
            for x, y in zip((k, v), got):                    # half a step of a code, 2^-4, or half of the least step 2^(e - 9), e <= -6 for |x| < 7
                assert torch.all((x - y[:, 0]).abs() <= torch.maximum(x.abs() * 2.0 ** -4, torch.tensor(2.0 ** -16, device="cuda")))
    for a, b in zip(*results):
        assert torch.equal(a, b)
