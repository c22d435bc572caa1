"""Sums of many equal weights in eora_cache_attention_rows: their roundings, all of one sign, do not add up over a long context.

All tokens but the first 64 have one score, a little above theirs, so that every weight is the same number with 24 bits, and lse and out are known.  A wavefront's lane adds up 32 (few rows: 16)
weights of each tile of keys, then the tiles: at most (32 + tiles + 8) 2^-24 of the sum.  The scores' fp32 product, its difference to the reference and the power of two: 2^-17 (1 + logit).  out is 1, of values
that are 1: its sum has a rounding for each 16 tokens and half of a weight, and its own rounding is 2^-11.  Added up weight by weight the sums over 131072 tokens are off by up to 6e-4 and 2e-4.
"""
import numpy as np
import pytest

from tests.test_gpu_attention_rows import gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,rows,heads,n", [(1, 128, 512, 131072), (1, 1000, 512, 8192), (300, 4, 8, 131072)])
def test_equal_weights(gpu, B, rows, heads, n):  # noqa: F811
    import torch
    dim, page, M = 64, 16, B * rows
    k, v = torch.zeros((2, 1, page, dim), device="cuda").half(), torch.ones((2, 1, page, dim), device="cuda").half()
    k[1, :, :, 0] = 1.0                                      # page 1: scores q[0]; page 0: 0
    score = torch.linspace(0.05, 2.7, M * heads, device="cuda").half().view(M, heads)
    q = torch.zeros((M, heads, dim), device="cuda").half()
    q[:, :, 0] = score
    table = torch.ones((B, n // page), dtype=torch.int32, device="cuda")
    table[:, :4] = 0
    lengths, starts = np.full(B, n, np.int32), np.arange(B + 1, dtype=np.int32) * rows
    narrow, _, b, _, _, _, _, parts, steps, _ = gpu.debug_attention_rows_unit(lengths, starts, M, heads, 1, dim, page, 16, n // page, 0, 0, 0)
    assert b == 0 and narrow == (B > 1) and parts == 1 and steps * (32 if narrow else 64) >= n - 1000
    out, lse = torch.empty_like(q), torch.empty((M, heads), device="cuda")
    gpu.cache_attention_rows(q, k, v, None, None, table, torch.from_numpy(lengths).cuda(), torch.from_numpy(starts).cuda(), out, lse, M, B, heads, 1, dim, heads * dim, 2, page, 16, 0,
                             n // page, 0, 0, 1.0, gpu.new_attention_rows_workspace(M, B, heads, 1, dim, n))
    torch.cuda.synchronize()
    s = score.double()
    seen = (torch.arange(M, device="cuda") % rows + n - rows + 1).double()[:, None]
    want = torch.log(64 + (seen - 64) * torch.exp(s))
    scores = 2.0 ** -17 * (1 + s)
    sums = (32 + (steps // 4 if narrow else steps) + 8) * 2.0 ** -24       # (few rows: four wavefronts share the tiles)
    assert bool(((lse.double() - want).abs() <= scores + sums).all()), ((lse.double() - want).abs() / (scores + sums)).max().item()
    assert bool(((out.double() - 1).abs() <= 2.0 ** -11 + (scores + sums + n / 8 * 2.0 ** -24)[..., None]).all())
