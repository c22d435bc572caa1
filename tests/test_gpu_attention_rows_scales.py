"""eora_cache_attention_rows with scales that are not finite, or 0: what a head's scale makes NaN is NaN for the rows that see a token, and nothing else changes."""
import numpy as np
import pytest

from tests.test_gpu_attention_rows import Rows, gpu  # noqa: F401
from tests.test_gpu_serving import TINY, U, close

pytestmark = pytest.mark.gpu


# requests whose first rows see nothing; tiles of 32 pairs and of 128; single tokens
@pytest.mark.parametrize("heads,single", [(4, False), (800, False), (4, True)])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_a_head_whose_scale_is_not_finite(gpu, heads, single, dim, value):  # noqa: F811
    requests = [(n, 1) for n in (0, 7, 150)] if single else [(0, 3), (40, 43), (150, 20)]

    def case():
        return Rows(72, requests, heads, 2, dim, "heads", 16, single=single)
    clean = case()
    base, base_lse = clean.run(gpu, 60, 2)
    sees = np.isfinite(base_lse[:, 0])
    assert 0 < sees.sum() < len(sees)
    of = slice(heads // 2, None)                             # query heads of kv head 1
    for what in ("ks", "vs"):
        c = case()
        getattr(c, what)[1] = value
        out, lse = c.run(gpu, 60, 2)
        assert np.array_equal(out[:, :heads // 2], base[:, :heads // 2]) and np.array_equal(lse[:, :heads // 2], base_lse[:, :heads // 2]), "the other kv head"
        assert not out[~sees].any() and np.all(lse[~sees] == -np.inf), "rows that see nothing"
        if what == "vs":
            assert not np.isfinite(out[sees, of]).any() and np.array_equal(lse, base_lse)
        elif np.isnan(value) or not single:
            assert np.isnan(out[sees, of]).all() and np.isnan(lse[sees, of]).all()


@pytest.mark.parametrize("heads", [4, 800])
@pytest.mark.parametrize("value", [np.inf, -np.inf])
def test_a_scale_of_zero_and_infinities(gpu, heads, value):  # noqa: F811
    """0 times an infinity is NaN, of a key for the rows that see it, of a query for its own row; all other scores are 0."""
    c = Rows(73, [(90, 60), (33, 33)], heads, 2, 64, "fp16", 16)
    p, o = c.place(0, 50)
    c.k[p, 1, o, 3] = value
    c.q[70, 0, 5] = value
    c.set()
    out, lse = c.run(gpu, scale=0.0)
    want, wl, size, _, _ = c.want(scale=0.0)
    assert np.isnan(wl[:60, heads // 2:]).sum() == 40 * heads // 2 and np.isnan(wl[70, 0])
    close(out, want, 1.25 * U * (np.abs(want) + size) + TINY, "out")
    close(lse, wl, 2.0 ** -17, "lse")
