"""GPU parity of eora_cache_attention_rows, both its forms, against the float64 definition of oracle/serving.py.

Tolerances, element by element (u = 2^-11: fp16's unit roundoff):
  out   1.25 u (|out| + sum p |v|) + tokens 2^-24 max|v| + 2^-25: a weight and the result are rounded to fp16 once each (single tokens: a weight has 20 bits), fp32 scores and
        sums, weights below 2^-36 of the largest may be lost
  lse   2^-17 (1 + largest sum |scale q k|): fp32 dot products
"""
import numpy as np
import pytest

from tests.test_gpu_serving import TINY, U, close

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


def stored(x, form, rng, kv):
    """(tensor, scales, float64 values) of a cache in a form; x: n_pages x kv x page x dim with NaN in unused places."""
    import torch

    from oracle import serving
    if form == "fp16":
        h = x.astype(np.float16)
        return dev(h), None, h.astype(np.float64)
    value = serving.e4m3_values()
    if form == "heads":
        s = rng.uniform(0.01, 0.03, kv).astype(np.float32)
        t = (dev(x) / dev(s)[:, None, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8)
        return t, dev(s), value[t.cpu().numpy()] * s.astype(np.float64)[:, None, None]
    n, kv, page, dim = x.shape
    blocks = np.nan_to_num(np.abs(x), nan=0.0, posinf=0.0).reshape(n, kv, page // 16, 16 * dim).max(-1)
    e = np.clip(np.ceil(np.log2(np.maximum(blocks, 1e-9) / 448)), -15, 8)
    by = np.repeat(2.0 ** e, 16, -1)[..., None]
    t = torch.from_numpy(np.clip(x / by, -448, 448)).float().to(torch.float8_e4m3fn).view(torch.uint8)
    byte = (e + 127).astype(np.uint8)
    byte[blocks == 0] = rng.choice([0, 255, 127], (blocks == 0).sum())          # unused blocks
    return t.cuda(), dev(byte), value[t.numpy()] * by


class Rows:
    """Requests of (tokens, rows) over a cache of random values whose unused places hold NaN, pages in any order; rows None: single tokens."""

    def __init__(self, seed, requests, heads, kv, dim, form, page, width=None, k_size=1.0, q_size=1.0, q_pad=0, tail=0, single=False):
        rng = self.rng = np.random.default_rng(seed)
        self.lengths = np.array([n for n, _ in requests], np.int32)
        self.starts = np.cumsum([0] + [r for _, r in requests]).astype(np.int32)
        self.single = single
        B = self.B = len(requests)
        used = [-(-max(0, n) // page) for n, _ in requests]
        self.width = max([1] + used) if width is None else width
        n_pages = self.n_pages = sum(used) + 2
        order = rng.permutation(n_pages)
        self.table = rng.choice(np.array([-1, n_pages, 2 ** 31 - 1, -2 ** 31]), (B, self.width)).astype(np.int32)
        self.k, self.v = np.full((n_pages, kv, page, dim), np.nan), np.full((n_pages, kv, page, dim), np.nan)
        at = 0
        for b, (n, _) in enumerate(requests):
            for p in range(used[b]):
                here = min(page, n - p * page)
                self.table[b, p] = order[at]
                self.k[order[at], :, :here] = rng.normal(0, k_size, (kv, here, dim))
                self.v[order[at], :, :here] = rng.normal(0, 1, (kv, here, dim))
                at += 1
        self.heads, self.kv, self.dim, self.form, self.page, self.q_pad = heads, kv, dim, form, page, q_pad
        self.M = int(self.starts[-1]) + tail
        self.q = rng.normal(0, q_size, (self.M, heads, dim)).astype(np.float16)
        self.set()

    def set(self):
        self.dk, self.ks, self.xk = stored(self.k, self.form, self.rng, self.kv)
        self.dv, self.vs, self.xv = stored(self.v, self.form, self.rng, self.kv)

    def place(self, b, t):
        """(page, token) of a request's token."""
        return self.table[b, t // self.page], t % self.page

    def run(self, eora, window=0, sinks=0, scale=None, ws=None, lse=True):
        import torch
        row = self.heads * self.dim + self.q_pad
        q = torch.full((self.M, row), np.nan, dtype=torch.float16, device="cuda")
        q[:, :self.heads * self.dim] = dev(self.q).view(self.M, -1)
        guard, size = 64, self.M * self.heads * self.dim
        buf = torch.full((size + 2 * guard,), 777.0, dtype=torch.float16, device="cuda")
        got = torch.full((self.M * self.heads + 8,), 777.0, dtype=torch.float32, device="cuda")
        ws = eora.new_attention_rows_workspace(self.M, self.B, self.heads, self.kv, self.dim, self.width * self.page) if ws is None else ws
        eora.cache_attention_rows(q, self.dk, self.dv, self.ks, self.vs, dev(self.table), dev(self.lengths), None if self.single else dev(self.starts), buf[guard:guard + size],
                                  got[4:-4] if lse else None, self.M, self.B, self.heads, self.kv, self.dim, row, self.n_pages, self.page, 16 if self.form == "fp16" else 8,
                                  16 if self.form == "blocks" else 0, self.width, window, sinks, self.dim ** -0.5 if scale is None else scale, ws)
        torch.cuda.synchronize()
        assert not ws[:49152].any(), "counters are left at zero"
        full, l = buf.cpu().numpy(), got.cpu().numpy()
        assert np.all(full[:guard] == 777.0) and np.all(full[guard + size:] == 777.0), "write outside out"
        assert np.all(l[:4] == 777.0) and np.all(l[-4:] == 777.0), "write outside lse"
        return full[guard:guard + size].reshape(self.M, self.heads, self.dim), l[4:-4].reshape(self.M, self.heads)

    def want(self, window=0, sinks=0, scale=None):
        from oracle import serving
        return serving.cache_attention_rows(self.q.astype(np.float64), self.xk, self.xv, self.table, self.lengths, None if self.single else self.starts, window, sinks,
                                            self.dim ** -0.5 if scale is None else scale)

    def check(self, eora, window=0, sinks=0, scale=None, **kw):
        out, lse = self.run(eora, window, sinks, scale, **kw)
        want, wl, size, most, logit = self.want(window, sinks, scale)
        used = int(self.starts[-1])
        assert np.all(out[used:] == 777.0) and np.all(lse[used:] == 777.0), "rows of no request were written"
        n = int(max(1, self.lengths.max(initial=0)))
        with np.errstate(invalid="ignore"):
            tol = 1.25 * U * (np.abs(want) + size) + n * 2.0 ** -24 * most[..., None] + TINY
        close(out[:used], want[:used], tol[:used], "out")
        close(lse[:used], wl[:used], 2.0 ** -17 * (1 + logit[:used]), "lse")
        return out[:used], lse[:used]


# tokens and rows
EDGES = [(1, 1), (2, 2), (15, 3), (16, 16), (17, 1), (31, 31), (32, 7), (33, 33), (63, 2), (64, 64), (65, 65), (127, 30), (128, 128), (129, 1), (130, 129), (200, 77)]
SHAPES = [
    # (tokens, rows) of the requests, heads, kv, dim, form, page
    ([(1, 1)], 1, 1, 64, "fp16", 16),
    ([(17, 17)], 32, 8, 128, "fp16", 16),
    ([(100, 40)], 8, 1, 256, "fp16", 16),
    (EDGES, 4, 2, 128, "fp16", 16),
    (EDGES, 4, 2, 128, "heads", 16),
    (EDGES, 4, 2, 128, "blocks", 16),
    (EDGES, 5, 1, 64, "blocks", 48),         # five query heads share keys: pairs of a row cross tiles
    (EDGES, 3, 3, 64, "fp16", 80),
    (EDGES, 2, 1, 256, "blocks", 32),
    (EDGES, 3, 3, 256, "heads", 16),
    ([(300, 300), (0, 0), (64, 0), (5, 5)], 7, 1, 64, "heads", 16),
    ([(0, 3), (2, 9), (40, 41)], 4, 2, 128, "fp16", 16),             # more rows than tokens: the first see nothing
    ([(2000, 3)], 4, 1, 128, "blocks", 64),  # few rows, many tokens: cut along the keys
    ([(1500, 200), (3, 3), (900, 1)], 3, 1, 64, "fp16", 16),
    ([(1200, 16)], 2, 2, 256, "fp16", 16),
    ([(40, 2)], 200, 1, 64, "fp16", 16),     # one row's heads are more than a tile
    ([(0, 0)], 4, 2, 64, "fp16", 16),
]


# many query heads: tiles of many pairs
MANY = [
    ([(300, 200), (77, 30), (1, 1), (64, 34)], 512, 1, 64, "fp16", 16),
    ([(257, 150), (40, 50), (120, 80)], 480, 2, 128, "fp16", 48),
    ([(130, 130), (900, 3), (200, 70)], 704, 1, 128, "blocks", 16),
    ([(100, 90), (350, 170)], 512, 4, 128, "heads", 32),
]


@pytest.mark.parametrize("requests,heads,kv,dim,form,page", MANY)
def test_many_pairs(gpu, requests, heads, kv, dim, form, page):
    c = Rows(heads + dim, requests, heads, kv, dim, form, page)
    assert c.M * heads >= 2 ** 17
    c.check(gpu)
    c.check(gpu, 50, 7)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", ["fp16", "heads", "blocks"])
@pytest.mark.parametrize("heads,kv,page", [(32, 2, 16), (45, 3, 48)])
def test_wide_tiles(gpu, dim, form, heads, kv, page):
    """Every length at which tiles of rows and keys begin and end, where there are rows enough for tiles of 128 pairs."""
    c = Rows(56 + dim, EDGES, heads, kv, dim, form, page, tail=1)
    assert c.M * heads > 96 * 128 and c.M * heads // kv > 64 * c.B
    c.check(gpu)
    c.check(gpu, 33, 20)


def test_many_pairs_cut_along_the_keys(gpu):
    """One long request among short ones, in tiles of 256 pairs."""
    Rows(54, [(3000, 3)] + [(10, 10)] * 50, 256, 1, 128, "blocks", 16).check(gpu)
    Rows(55, [(2000, 2)] + [(7, 7)] * 75, 256, 1, 64, "fp16", 16).check(gpu, 900, 5)


@pytest.mark.parametrize("requests,heads,kv,dim,form,page", SHAPES)
def test_shapes(gpu, requests, heads, kv, dim, form, page):
    c = Rows(len(requests) + heads + dim, requests, heads, kv, dim, form, page, tail=2)
    c.check(gpu)
    out = c.run(gpu)[0]
    again = c.run(gpu, lse=False)[0]
    assert np.array_equal(out.view(np.uint16), again.view(np.uint16)), "a second time, or without lse, other bits"


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (16, 1), (31, 0), (40, 64), (64, 37), (100, 4), (3, 10 ** 9), (10 ** 9, 3)])
@pytest.mark.parametrize("form,dim", [("fp16", 64), ("blocks", 128), ("heads", 256)])
def test_window_and_first_tokens(gpu, window, sinks, form, dim):
    Rows(31, [(n, min(n, 90)) for n, _ in EDGES] + [(500, 5), (333, 333)], 2, 1, dim, form, 16).check(gpu, window, sinks)


SINGLE = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 200]


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 9), (1, 0), (1, 1), (16, 1), (16, 40), (31, 32), (50, 33), (64, 37), (100, 4), (3, 10 ** 9)])
@pytest.mark.parametrize("heads,kv,dim,form,page", [(8, 2, 128, "blocks", 16), (5, 5, 64, "fp16", 48), (6, 1, 64, "heads", 80), (3, 3, 256, "blocks", 32), (20, 1, 64, "blocks", 16)])
def test_single_tokens(gpu, window, sinks, heads, kv, dim, form, page):
    c = Rows(32 + heads, [(n, 1) for n in SINGLE + [700, 5, 1100]], heads, kv, dim, form, page, single=True)
    c.check(gpu, window, sinks)


@pytest.mark.parametrize("form", ["fp16", "heads", "blocks"])
def test_single_tokens_and_rows_of_one_agree(gpu, form):
    """The two forms, on requests with a row each: within their tolerances of one definition, and of each other within the sum of them."""
    c = Rows(33, [(n, 1) for n in SINGLE[1:] + [3000]], 8, 2, 128, form, 16)
    a = c.check(gpu, 100, 5)[0]
    c.single = True
    b = c.check(gpu, 100, 5)[0]
    assert np.abs(a.astype(np.float64) - b).max() < 0.01


def test_without_first_tokens_the_bits_of_the_single_token_call(gpu):
    """Windows alone and scales by head are eora_cache_attention()."""
    import torch
    for form in ("fp16", "heads"):
        c = Rows(34, [(n, 1) for n in SINGLE], 8, 2, 64, form, 16, single=True)
        for window in (0, 40):
            got = c.run(gpu, window)[0]
            out = torch.empty((c.M, 8, 64), dtype=torch.float16, device="cuda")
            gpu.cache_attention(dev(c.q), c.dk, c.dv, c.ks, c.vs, dev(c.table), dev(c.lengths), out, None, c.B, 8, 2, 64, 512, c.n_pages, 16, 16 if form == "fp16" else 8, c.width,
                                window, 0.125, gpu.new_attention_workspace(c.B, 8, 2, 64, c.width * 16))
            assert np.array_equal(out.cpu().numpy().view(np.uint16), got.view(np.uint16))


def test_many_requests(gpu):
    """More requests than a workgroup has threads."""
    rng = np.random.default_rng(35)
    sizes = [(int(n), int(rng.integers(0, min(n, 4) + 1))) for n in rng.integers(0, 40, 700)]
    Rows(36, sizes, 2, 1, 64, "fp16", 16).check(gpu)
    Rows(36, [(n, 1) for n, _ in sizes], 2, 1, 64, "blocks", 16, single=True).check(gpu, 9, 3)


@pytest.mark.parametrize("requests, heads, kv, dim, form", [
    ([(40 + i % 7, 33 + i % 9) for i in range(66)], 8, 2, 64, "fp16"),                                     # tiles of many rows
    ([(60, 40)] * 40 + [(900, 90)] + [(5, 0), (0, 0)] * 10 + [(1500, 1)] * 9, 8, 2, 128, "blocks"),        # some of them cut along the keys
    ([(20, 2)] * 68 + [(9000, 3)] + [(30, 1)] * 5, 4, 1, 64, "fp16"),                                       # few rows, one request cut
    ([(i % 5, i % 3) for i in range(4170)], 2, 1, 64, "fp16"),                                              # more than 64 in each of 64 stretches
    ([(3, 1)] * 65, 1, 1, 256, "heads")])
def test_more_requests_than_a_wavefront_plans(gpu, requests, heads, kv, dim, form):
    Rows(61, requests, heads, kv, dim, form, 16).check(gpu)


def test_lengths_beyond_the_table_and_missing_pages(gpu):
    for dim, form in ((64, "fp16"), (128, "blocks"), (256, "heads")):
        c = Rows(37, [(90, 50), (64, 3), (33, 33), (50, 20)], 4, 2, dim, form, 16, width=6)
        c.lengths[:] = [90, -7, 33, 50]
        c.table[2, 1] = -1                   # tokens 16 .. 31 of the third request are masked
        c.table[3] = 10 ** 9                 # the last one has no page at all
        out, lse = c.check(gpu)
        assert not out[50:53].any() and not out[86:].any() and np.all(lse[50:53] == -np.inf)
        c.check(gpu, 20, 3)
        c = Rows(38, [(96, 20), (64, 9)], 4, 2, dim, form, 16, width=6)
        full = c.want()
        c.lengths[0] = 2 ** 31 - 1           # as far as the table goes
        out, _ = c.run(gpu)
        close(out, full[0], 1.25 * U * (np.abs(full[0]) + full[2]) + 1e-4, "out")


def test_starts_out_of_range_and_requests_without_rows(gpu):
    """Rows that there are not are not read or written."""
    c = Rows(39, [(40, 10), (50, 10), (60, 10)], 4, 2, 64, "fp16", 16)
    c.starts[:] = [-5, 10, 10, 2 ** 30]
    want = c.want()
    out, _ = c.run(gpu)
    close(out, want[0], 1.25 * U * (np.abs(want[0]) + want[2]) + 1e-4, "out")
    c.starts[:] = [4, 9, 3, 20]              # decreasing: the second request has none; the others as they say
    out, _ = c.run(gpu)
    assert np.all(out[20:] == 777.0) and np.all(out[:3] == 777.0)


def test_rising_scores_and_large_ones(gpu):
    for dim, form in ((128, "fp16"), (64, "blocks"), (256, "fp16")):
        c = Rows(40, [(1500, 20), (300, 300)], 4, 1, dim, form, 16)
        for b in range(2):
            for t in range(c.lengths[b]):
                p, o = c.place(b, t)
                c.k[p, :, o] = c.q[c.starts[b + 1] - 1].mean(0) * (t / 200.0) + 0.1 * c.k[p, :, o]
        c.set()
        c.check(gpu, scale=0.5)
    Rows(41, [(600, 33), (33, 33)], 8, 2, 64, "fp16", 16, k_size=8.0, q_size=8.0).check(gpu)
    for form in ("fp16", "heads"):
        c = Rows(42, [(300, 40)], 4, 1, 64, form, 16)
        c.check(gpu, scale=0.0)              # all weights alike
        c.check(gpu, scale=-0.25)


def test_many_tokens_far_below_the_largest(gpu):
    """4000 tokens 16 nats below one have their part."""
    c = Rows(43, [(4001, 3)], 2, 1, 64, "fp16", 16)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    c.k[:, :, :, 0] = np.where(np.isnan(c.k[:, :, :, 0]), np.nan, 0)
    p, o = c.place(0, 0)
    c.k[p, 0, o, 0] = 16
    c.v = np.where(np.isnan(c.v), np.nan, 1000.0)
    c.v[p, 0, o] = 0
    c.set()
    c.check(gpu, scale=1.0)


@pytest.mark.parametrize("dim,pairs", [(64, 1), (128, 1), (256, 1), (64, 194), (128, 194)])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_what_a_row_does_not_see_is_not_used(gpu, dim, pairs, value):
    """Keys and values that are not finite, of tokens that some rows of a tile see and others do not: rows that do not see them have the bits that they have without them."""
    heads = 4 * pairs

    def case():
        return Rows(44, [(150, 100), (70, 70)], heads, 2, dim, "fp16", 16)
    clean = case()
    base, base_lse = clean.run(gpu, 60, 2)
    for what in ("k", "v"):
        c = case()
        for b, t in ((0, 75), (1, 30), (1, 0)):
            p, o = c.place(b, t)
            getattr(c, what)[p, 1, o, 5] = value
        c.set()
        out, lse = c.run(gpu, 60, 2)
        want = c.want(60, 2)[0]
        for b in range(2):
            for r in range(c.starts[b], c.starts[b + 1]):
                p = c.lengths[b] - c.starts[b + 1] + r
                hit = any(t <= p and (t > p - 60 or t < 2) for at, t in ((0, 75), (1, 30), (1, 0)) if at == b)
                assert np.array_equal(out[r, :heads // 2], base[r, :heads // 2]), "the other kv head"
                if not hit:
                    assert np.array_equal(out[r], base[r]) and np.array_equal(lse[r], base_lse[r]), "row %d of request %d" % (r, b)
                elif what == "v":
                    for i in (heads // 2, heads - 1):
                        close(out[r, i, 5], want[r, i, 5], 0, "row %d" % r)
                        assert np.array_equal(np.delete(out[r, i], 5), np.delete(base[r, i], 5))


def test_a_score_of_minus_infinity_masks_its_token(gpu):
    c = Rows(45, [(70, 20)], 2, 2, 64, "fp16", 16)
    c.q = np.abs(c.q)
    p, o = c.place(0, 13)
    c.k[p, 0, o] = -np.inf
    c.set()
    c.check(gpu)


def test_rows_of_a_wider_buffer(gpu):
    Rows(46, [(50, 30), (20, 20)], 4, 2, 128, "fp16", 16, q_pad=72).check(gpu)


def test_pieces_of_a_prompt_are_the_whole(gpu):
    """A prompt at once, and by pieces: each row's result is the same, whatever it is computed beside."""
    c = Rows(47, [(300, 300)], 4, 2, 128, "blocks", 16)
    whole, lse = c.check(gpu)
    at = 0
    for n in (1, 63, 100, 136):
        part = Rows(47, [(300, 300)], 4, 2, 128, "blocks", 16)
        part.q, part.M, part.starts = part.q[at:at + n], n, np.array([0, n], np.int32)
        part.lengths[:] = at + n
        out, l = part.run(gpu)
        assert np.abs(out.astype(np.float64) - whole[at:at + n]).max() < 0.01 and np.abs(l - lse[at:at + n]).max() < 1e-4
        at += n


def test_one_workspace_for_calls_of_every_kind(gpu):
    """Cut and uncut prompts, single tokens, the call without first tokens, one after the other: all leave it usable."""
    import torch
    ws = gpu.new_attention_rows_workspace(400, 20, 16, 2, 256, 8192)
    ws[49152:] = 0xAB
    for seed in range(3):
        Rows(48 + seed, [(3000, 5), (20, 20)], 4, 2, 128, "fp16", 16).check(gpu, ws=ws)
        Rows(48 + seed, [(n, 1) for n in (3000, 5, 900)], 8, 2, 64, "blocks", 16, single=True).check(gpu, ws=ws)
        Rows(48 + seed, [(2000, 100)], 4, 1, 256, "blocks", 32).check(gpu, 700, 9, ws=ws)
        Rows(48 + seed, [(2000, 1)], 4, 1, 64, "fp16", 32, single=True).check(gpu, ws=ws)
    assert torch.cuda.is_available()


def test_beyond_32_bits(gpu):
    """Pages behind 2^32 elements of a pool."""
    import torch
    for single in (False, True):
        c = Rows(52, [(40, 1), (17, 1)] if single else [(40, 30), (17, 2)], 4, 2, 64, "blocks", 16, single=single)
        out, lse = c.run(gpu)
        n = 2 ** 32 // (2 * 16 * 64) + 7
        big = [torch.empty((n, 2, 16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
        bytes_ = [torch.empty((n, 2, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
        for t, small in zip(big + bytes_, (c.dk, c.dv, c.ks, c.vs)):
            t[n - c.n_pages:] = small
        c.dk, c.dv, c.ks, c.vs = big + bytes_
        c.table = np.where((c.table >= 0) & (c.table < c.n_pages), c.table + n - c.n_pages, -1).astype(np.int32)
        c.n_pages = n
        got = c.run(gpu)
        assert np.array_equal(got[0].view(np.uint16), out.view(np.uint16)) and np.array_equal(got[1], lse)


def test_together_on_another_stream_and_in_a_graph(gpu):
    """A prompt and a token after it: stored with scales by block, attended to, read back; eager, on a stream of its own, captured and replayed with work between: the eager bits."""
    import torch
    heads, kv, dim, page, P = 8, 2, 128, 32, 75
    rng = np.random.default_rng(53)
    rows = lambda n, h: dev(rng.normal(0, 1, (n, h, dim)).astype(np.float16))      # noqa: E731
    qp, kp, vp, qt, kt, vt = rows(P, heads), rows(P, kv), rows(P, kv), rows(1, heads), rows(1, kv), rows(1, kv)
    table = torch.tensor([[4, 1, 3]], dtype=torch.int32, device="cuda")
    at = torch.arange(P + 1, device="cuda")
    slots = table[0, at // page].long() * page + at % page
    codes, scales = [torch.zeros((5, kv, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)], [torch.zeros((5, kv, page // 16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    op, ot, back = torch.empty_like(qp), torch.empty_like(qt), [torch.empty((P + 1, kv, dim), dtype=torch.float16, device="cuda") for _ in range(2)]
    starts, n0, n1 = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, P], [P], [P + 1]))
    ws = gpu.new_attention_rows_workspace(P, 1, heads, kv, dim, 96)

    def step():
        for t in codes + scales:
            t.zero_()
        gpu.cache_append_blocks(qp, kp, vp, None, None, None, None, slots[:P], qp, *codes, *scales, P, heads, kv, dim, heads * dim, kv * dim, kv * dim, 0, False, 0, 0.0, 5, page)
        gpu.cache_attention_rows(qp, *codes, *scales, table, n0, starts, op, None, P, 1, heads, kv, dim, heads * dim, 5, page, 8, 16, 3, 0, 0, 0.1, ws)
        gpu.cache_append_blocks(qt, kt, vt, None, None, None, None, slots[P:], qt, *codes, *scales, 1, heads, kv, dim, heads * dim, kv * dim, kv * dim, 0, False, 0, 0.0, 5, page)
        gpu.cache_attention_rows(qt, *codes, *scales, table, n1, None, ot, None, 1, 1, heads, kv, dim, heads * dim, 5, page, 8, 16, 3, 40, 4, 0.1, ws)
        gpu.cache_read(*codes, *scales, slots, *back, P + 1, kv, dim, 5, page, 8, 16)

    step()
    torch.cuda.synchronize()
    outs = [op, ot] + back
    want = [t.clone() for t in outs]
    # against the definition, from what is read back
    from oracle import serving
    k, v = (np.zeros((5, kv, page, dim)) for _ in range(2))
    for t, s in enumerate(slots.tolist()):
        k[s // page, :, s % page], v[s // page, :, s % page] = back[0][t].double().cpu().numpy(), back[1][t].double().cpu().numpy()
    for q, o, n, st, window, sinks in ((qp, op, P, [0, P], 0, 0), (qt, ot, P + 1, None, 40, 4)):
        ref = serving.cache_attention_rows(q.double().cpu().numpy(), k, v, table.cpu().numpy(), [n], st, window, sinks, float(np.float32(0.1)))
        close(o.cpu().numpy(), ref[0], 1.25 * U * (np.abs(ref[0]) + ref[2]) + n * 2.0 ** -24 * ref[3][..., None] + TINY, "out")
    assert (back[0][:P].float() - kp.float()).abs().max() <= 2.0 ** -4 * 8
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for t in outs:
            t.zero_()
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        step()                               # eager work between the replays, in the same workspace


@pytest.mark.parametrize("B", [7, 70])
def test_a_captured_call_follows_lengths_and_rows(gpu, B):
    """Lengths and rows are read on the device: a captured call takes those of each replay, and gives the eager bits; so it does where other calls use the workspace between."""
    import torch
    heads, kv, dim, page, width, M = 8, 2, 128, 16, 20, 40 * B
    torch.manual_seed(B)
    q = torch.randn((M, heads, dim), device="cuda").half()
    k, v = (torch.randn((B * width, kv, page, dim), device="cuda").half() for _ in range(2))
    table = torch.randperm(B * width, device="cuda").int().view(B, width)
    lengths, starts = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    ws = gpu.new_attention_rows_workspace(M, B, heads, kv, dim, width * page)

    def call(out, n=lengths, s=starts):
        gpu.cache_attention_rows(q, k, v, None, None, table, n, s, out, None, M, B, heads, kv, dim, heads * dim, B * width, page, 16, 0, width, 0, 0, 0.1, ws)

    rng = np.random.default_rng(B)
    held = torch.full_like(q, 7.0)
    call(held)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(held)
    for _ in range(4):
        n = rng.integers(1, width * page + 1, B)
        s = np.concatenate([[0], np.cumsum(np.minimum(rng.integers(0, 41, B), n))])
        lengths.copy_(torch.from_numpy(n.astype(np.int32)))
        starts.copy_(torch.from_numpy(s.astype(np.int32)))
        want = torch.full_like(q, 7.0)
        call(want, lengths.clone(), starts.clone())
        held.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want) and bool((want[:int(s[-1])] != 7.0).any()) and bool((want[int(s[-1]):] == 7.0).all())
        assert not ws[:49152].any()
