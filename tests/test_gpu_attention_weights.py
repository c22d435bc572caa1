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


@pytest.mark.parametrize("tokens", [4001, 131072])
@pytest.mark.parametrize("ahead", [10.0, 14.0, 16.0, 17.0])
@pytest.mark.parametrize("bits", [16, 8])
def test_one_token_far_above_many(gpu, bits, ahead, tokens):
    """The first token's score is `ahead` above those of all others, which are alike, and its value is zero: what is left is the others' part.
    A weight's absolute error, which counts where it is far below the largest, is at most 2^-36 of that."""
    import torch
    heads, dim, page = 2, 64, 64
    n_pages = -(-tokens // page)
    q = torch.full((1, heads, dim), 0.5, device="cuda").half()
    k = torch.zeros((n_pages, 1, page, dim), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    v = torch.randint(1, 8, (n_pages, 1, page, dim), generator=g, device="cuda") * 0.25      # exact in 8 bits too
    k[0, 0, 0] = 1.0
    v[0, 0, 0] = 0.0
    scale = ahead / (0.5 * dim)
    kind = torch.float16 if bits == 16 else torch.float8_e4m3fn
    one = torch.ones(1, device="cuda") if bits == 8 else None
    out, lse = torch.full((1, heads, dim), 7.0, device="cuda").half(), torch.zeros((1, heads), device="cuda")
    ws = gpu.new_attention_workspace(1, heads, 1, dim, n_pages * page)
    gpu.cache_attention(q, k.to(kind), v.to(kind), one, one, torch.arange(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([tokens], dtype=torch.int32, device="cuda"),
                        out, lse, 1, heads, 1, dim, heads * dim, n_pages, page, bits, n_pages, 0, scale, ws)
    torch.cuda.synchronize()
    others = v.double().view(-1, dim)[:tokens].cpu().numpy()
    w = np.exp(-ahead)
    total = 1 + (tokens - 1) * w
    want = w * others.sum(0) / total
    got = out[0].double().cpu().numpy()
    # U: the result; the scores and their difference in fp32; halves of a weight; its absolute error, of `tokens` weights of a value of 1.75 at most
    tol = (U + 2.0 ** -17 * (1 + ahead)) * want + tokens * 2.0 ** -36 * 1.75 / total + TINY
    assert np.all(np.abs(got - want) <= tol), "off by %.3g of itself" % np.abs(got / want - 1).max()
    assert np.all(np.abs(lse.cpu().numpy() - (ahead + np.log(total))) <= 2.0 ** -17 * (1 + ahead))
