"""Weights of eora_cache_attention_rows with several rows a request keep 20 bits on their way to the values.

A row that sees a few tokens has an out that the values nearly cancel in: what its own rounding leaves then is what the weights lost.  Tolerance (u = 2^-11):
  u |out|                         the result, rounded once
  2^-17 (1 + logit) sum p |v|     a weight: two fp16 cut off its first 20 bits (2^-20), its score an fp32 dot product and a product with the scale, subtracted from a reference of up to 15 in fp32
                                  (2^-18 of the score's parts and of 1), the hardware's power of two (2^-22); the same for the sum that out is divided by
  2^-25                           half of fp16's least step
With weights of 11 bits an element is off by up to 2^-12 sum p |v| beside u |out|, 16 times the second term for a logit of 1.
"""
import numpy as np
import pytest

from tests.test_gpu_attention_rows import Rows, gpu  # noqa: F401
from tests.test_gpu_serving import TINY, U, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,dim", [("fp16", 64), ("fp16", 128), ("fp16", 256), ("blocks", 128), ("heads", 64), ("blocks", 256)])
@pytest.mark.parametrize("heads,kv", [(4, 2), (400, 1)])     # tiles of 32 pairs, of 128
def test_few_tokens_whose_values_cancel(gpu, form, dim, heads, kv):  # noqa: F811
    c = Rows(70 + dim + heads, [(150, 100), (5, 5), (64, 33)], heads, kv, dim, form, 16, q_size=0.5, k_size=0.5)
    for window, sinks in ((3, 0), (1, 1), (0, 0)):
        out, lse = c.run(gpu, window, sinks)
        want, wl, size, _, logit = c.want(window, sinks)
        close(out, want, U * np.abs(want) + 2.0 ** -17 * (1 + logit[..., None]) * size + TINY, "out")
        close(lse, wl, 2.0 ** -17 * (1 + logit), "lse")


def test_one_token_far_above_the_others(gpu):  # noqa: F811
    """Scores that rise by less than the reference does: the last token has nearly all of the weight, and out is nearly its value."""
    c = Rows(71, [(40, 8)], 8, 2, 64, "fp16", 16)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    p, o = zip(*(c.place(0, t) for t in range(40)))
    c.k[p, :, o, 0] = np.linspace(0, 2.5, 40)[:, None]
    c.k[p, :, o, 1:] = 0
    c.set()
    for window in (1, 2, 20):
        out = c.run(gpu, window, 0, scale=1.0)[0]
        want, _, size, _, logit = c.want(window, 0, scale=1.0)
        close(out, want, U * np.abs(want) + 2.0 ** -17 * (1 + logit[..., None]) * size + TINY, "out")
