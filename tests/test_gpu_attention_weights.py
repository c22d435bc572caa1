"""eora_cache_attention where the softmax weights' own rounding shows: values that cancel, so that little is left of the sum but the errors of its
terms.

Tolerance, element by element (u = 2^-11: fp16's unit roundoff; L: largest sum of |scale q k| of a row):
  u |out| + 2^-17 (1 + L) sum p |v| + 2^-25: one rounding of the result; a score's error is at most 2^-20 L of its fp32 dot product and 2^-22 L of the
  scaling, a weight's beside it a few 2^-24 of exp2 and 2^-20.7 of its two halves: 2^-19 (1 + L) together, once in the sum over v and once in the sum
  of weights, and fp32 sums in chains of at most some 100 additions.
"""
import numpy as np
import pytest

from tests.test_gpu_serving import Cache, close

pytestmark = pytest.mark.gpu

U = 2.0 ** -11
TINY = 2.0 ** -25


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lengths,heads,kv,dim,page", [
    ([2, 4, 6, 32, 64], 4, 2, 64, 16),
    ([2, 34, 100, 700], 8, 2, 128, 16),
    ([4, 40, 300], 5, 5, 256, 48),
    ([3000], 16, 1, 128, 16),                # parts of several workgroups
])
def test_values_that_cancel(gpu, lengths, heads, kv, dim, page, bits):
    """Every second token has the key of the one before it, a little off, and its value negated."""
    from oracle import serving
    c = Cache(len(lengths) + dim + bits, lengths, heads, kv, dim, bits, page, k_size=0.5, q_size=0.25)
    rng = np.random.default_rng(dim + bits)
    for b, n in enumerate(lengths):
        for t in range(1, n, 2):
            at, was = (c.table[b, t // page], slice(None), t % page), (c.table[b, (t - 1) // page], slice(None), (t - 1) % page)
            c.k[at] = c.k[was] + 0.1 * rng.normal(0, 1, (kv, dim))
            c.v[at] = -c.v[was]
    c.set(np.random.default_rng(3))
    out, lse = c.run(gpu)
    want, wl, size, _, logit = serving.cache_attention(c.q.astype(np.float64), c.k, c.v, c.table, c.lengths, 0, dim ** -0.5)
    close(out, want, U * np.abs(want) + 2.0 ** -17 * (1 + logit[..., None]) * size + TINY, "out")
    close(lse, wl, 2.0 ** -17 * (1 + logit), "lse")
