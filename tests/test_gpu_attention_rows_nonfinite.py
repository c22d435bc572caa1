"""Keys and values that are not finite in eora_cache_attention_rows: caches of 8 bits (NaN codes), and tiles of rows that are cut along the keys (their parts are joined).

Rows that do not see such a token, and the other kv head, have the bits that they have without it.  A NaN key makes a row that sees it NaN; a value makes its column NaN or the infinity, and
leaves the row's other columns as they are."""
import numpy as np
import pytest

from tests.test_gpu_attention_rows import Rows, gpu  # noqa: F401

pytestmark = pytest.mark.gpu
COLUMN = 5


def plant(c, what, b, t, value):
    """A key's or value's column of a token, in kv head 1: a NaN code, or an fp16 value."""
    p, o = c.place(b, t)
    pages = c.dk if what == "k" else c.dv
    pages[int(p), 1, int(o), COLUMN] = value if c.form == "fp16" else 0x7F if t % 2 else 0xFF


def check(gpu, case, tokens, values, window, sinks):  # noqa: F811
    """tokens: (request, token) that are planted."""
    clean = case()
    base, base_lse = clean.run(gpu, window, sinks)
    half = clean.heads // 2
    assert np.isfinite(base).all()
    for value in values:
        for what in "kv":
            c = case()
            for b, t in tokens:
                plant(c, what, b, t, value)
            out, lse = c.run(gpu, window, sinks)
            assert np.array_equal(out[:, :half], base[:, :half]) and np.array_equal(lse[:, :half], base_lse[:, :half]), "the other kv head"
            hits = 0
            for b in range(c.B):
                for r in range(int(c.starts[b]), int(c.starts[b + 1])):
                    p = int(c.lengths[b] - c.starts[b + 1]) + r
                    hit = any(at == b and t <= p and (not window or t > p - window or t < sinks) for at, t in tokens)
                    hits += hit
                    if not hit:
                        assert np.array_equal(out[r], base[r]) and np.array_equal(lse[r], base_lse[r]), "row %d of request %d" % (r, b)
                    elif what == "v":
                        got = out[r, half:, COLUMN]
                        assert np.isnan(got).all() if np.isnan(value) else np.all(got == value), "row %d of request %d" % (r, b)
                        assert np.array_equal(np.delete(out[r, half:], COLUMN, -1), np.delete(base[r, half:], COLUMN, -1)) and np.array_equal(lse[r], base_lse[r])
                    elif np.isnan(value):
                        assert np.isnan(out[r, half:]).all() and np.isnan(lse[r, half:]).all(), "row %d of request %d" % (r, b)
            assert hits > 0


@pytest.mark.parametrize("form", ["heads", "blocks"])
@pytest.mark.parametrize("dim,heads", [(64, 4), (128, 4), (256, 4), (64, 776), (128, 776), (256, 776)])     # tiles of 32 pairs, of 128
def test_codes_that_are_nan(gpu, form, dim, heads):  # noqa: F811
    def case():
        return Rows(90 + dim, [(150, 100), (70, 70)], heads, 2, dim, form, 16)
    check(gpu, case, ((0, 75), (1, 30), (1, 0), (1, 69)), [np.nan], 60, 2)


@pytest.mark.parametrize("form", ["fp16", "heads", "blocks"])
@pytest.mark.parametrize("requests,heads,dim", [([(2500, 40)], 4, 64), ([(2500, 40), (30, 30)], 4, 128), ([(2600, 8)], 8, 256),                        # few rows
                                                ([(2500, 300)], 64, 128), ([(2700, 250), (20, 3)], 80, 64), ([(2500, 300)], 32, 256)])                # many
def test_in_parts_of_a_tile(gpu, requests, heads, dim, form):  # noqa: F811
    """At the window's edge, which is in a tile's first part, on the diagonal, in its last, and between."""
    (n, rows), window = requests[0], 1900

    def case():
        return Rows(91 + dim, requests, heads, 2, dim, form, 16)
    c = case()
    got = [gpu.debug_attention_rows_unit(c.lengths, c.starts, c.M, c.heads, c.kv, c.dim, c.page, 16 if form == "fp16" else 8, c.width, window, 3, i) for i in range(8)]
    assert max(g[7] for g in got) > 1
    edge = n - rows - window + rows // 2                     # the first half of the rows see it
    for tokens in (((0, edge),), ((0, n - 2),), ((0, edge), (0, edge + 1), (0, n - rows // 2))):
        check(gpu, case, tokens, [np.nan, np.inf] if form == "fp16" else [np.nan], window, 3)
