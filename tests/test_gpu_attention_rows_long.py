"""eora_cache_attention_rows where a workgroup goes through many tiles of keys: what it looks up of the page table is replaced on the way, every 16 tiles of 64 keys for many rows, every 32 of a wavefront's
tiles of 32 for few.  Against the float64 definition, with the tolerances of tests/test_gpu_attention_rows.py; the plan is asked for on the host, so that no case is cut into parts too short."""
import numpy as np
import pytest

from tests.test_gpu_attention_rows import Rows, gpu  # noqa: F401
from tests.test_gpu_serving import TINY, U, close

pytestmark = pytest.mark.gpu


def steps_of(eora, c, window, sinks):
    """(few rows, parts, tiles of keys) of the first workgroup: the last tile of a request's rows."""
    got = eora.debug_attention_rows_unit(c.lengths, c.starts, c.M, c.heads, c.kv, c.dim, c.page, 16 if c.form == "fp16" else 8, c.width, window, sinks, 0)
    return bool(got[0]), got[7], got[8]


def lose_pages(c, *tokens):
    """The pages of some tokens are no longer there."""
    for t in tokens:
        c.table[:, t // c.page] = -1


@pytest.mark.parametrize("heads,kv,dim,form,page", [(4096, 1, 64, "fp16", 16), (4096, 2, 128, "fp16", 48), (4096, 1, 128, "blocks", 16), (4096, 2, 64, "heads", 32), (4096, 1, 128, "heads", 16),
                                                    (2048, 1, 256, "fp16", 16), (2048, 2, 256, "blocks", 32)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1300, 100), (1100, 1000), (2000, 5)])
def test_many_rows(gpu, heads, kv, dim, form, page, window, sinks):  # noqa: F811
    c = Rows(80 + dim + kv, [(3000, 16)], heads, kv, dim, form, page)
    lose_pages(c, 1000, 1030, 2050, 2400)
    narrow, parts, steps = steps_of(gpu, c, window, sinks)
    assert not narrow and parts == 1 and steps > (20 if window else 40)
    c.check(gpu, window, sinks)


def shared(seed, B, n, rows, heads, kv, dim, form, page):
    """B requests of up to n tokens, over the same pages in other orders."""
    c = Rows(seed, [(n, rows)], heads, kv, dim, form, page)
    assert n % page == 0
    c.B, c.M = B, B * rows
    c.table = np.stack([c.rng.permutation(c.table[0]) for _ in range(B)])
    c.lengths = (n - c.rng.integers(0, 2 * page, B)).astype(np.int32)
    c.starts = (np.arange(B + 1) * rows).astype(np.int32)
    c.q = c.rng.normal(0, 1, (c.M, heads, dim)).astype(np.float16)
    return c


@pytest.mark.parametrize("heads,kv,dim,form,page", [(4, 1, 64, "fp16", 16), (8, 2, 128, "blocks", 16), (3, 1, 128, "heads", 48), (2, 1, 128, "fp16", 16), (4, 1, 256, "blocks", 32), (5, 1, 64, "blocks", 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (8900, 1100), (9000, 40)])
def test_few_rows(gpu, heads, kv, dim, form, page, window, sinks):  # noqa: F811
    from oracle import serving
    B, rows = 300 // kv, 3
    c = shared(81 + dim, B, 10080, rows, heads, kv, dim, form, page)
    lose_pages(c, 4100, 4200, 8200, 8300)
    narrow, parts, steps = steps_of(gpu, c, window, sinks)
    assert narrow and parts == 1 and steps // 4 > 64
    out, lse = c.run(gpu, window, sinks)
    for b in (0, 1, 63, 64, B // 2, B - 1):
        at = slice(int(c.starts[b]), int(c.starts[b + 1]))
        want, wl, size, most, logit = serving.cache_attention_rows(c.q[at].astype(np.float64), c.xk, c.xv, c.table[b:b + 1], c.lengths[b:b + 1], [0, rows], window, sinks, dim ** -0.5)
        close(out[at], want, 1.25 * U * (np.abs(want) + size) + c.lengths[b] * 2.0 ** -24 * most[..., None] + TINY, "out of request %d" % b)
        close(lse[at], wl, 2.0 ** -17 * (1 + logit), "lse of request %d" % b)


@pytest.mark.parametrize("requests,heads,kv,dim,form", [([(40, 40)], 8, 2, 64, "fp16"), ([(512, 512)], 16, 2, 128, "blocks"), ([(300, 200), (5, 5), (0, 0)], 32, 4, 64, "heads"),
                                                        ([(300, 3), (17, 17), (64, 1)], 6, 2, 128, "fp16"), ([(90, 60), (33, 33)], 4, 1, 256, "blocks"), ([(700, 90)] + [(30, 2)] * 70, 16, 2, 64, "fp16")])
def test_a_table_with_much_more_room(gpu, requests, heads, kv, dim, form):  # noqa: F811
    """Room for 131072 tokens, as a server's table has: the same requests, whatever tiles they then have."""
    for width in (129, 8192):
        c = Rows(82 + dim, requests, heads, kv, dim, form, 16, width=width)
        c.check(gpu)
        c.check(gpu, 100, 9)
