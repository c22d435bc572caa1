"""eora_cache_attention's workspace: no larger than what the workgroups of a launch can fill, not written beyond, and zero in its first 48 KiB only."""
import pytest

import paper_2410_21271_amd as eora

HEAD = 48 << 10


def test_no_larger_than_a_launch_can_fill():
    """Two results of (dim + 2) fp32 a row of 4 wavefronts in 768, 512 or 256 workgroups, whichever of the widths up to this one takes most."""
    size = eora.cache_attention_workspace_bytes
    for heads, kv, rows in ((8, 8, 1), (8, 2, 4), (16, 1, 16), (40, 2, 16)):
        for dim, words in ((64, 768 * 66), (128, 512 * 130), (256, 512 * 130)):
            assert HEAD + 32 * words * rows <= size(64, heads, kv, dim, 4096) <= HEAD + 32 * words * rows + 256
    assert size(1, 16, 1, 256, 100) < 35e6


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv,dim,bits", [(13, 13, 64, 16), (8, 2, 128, 16), (16, 1, 256, 8), (17, 1, 256, 16), (6, 3, 128, 8)])
def test_filled_with_anything_behind_the_counters(heads, kv, dim, bits):
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    page, lengths = 16, [1, 5000, 37, 900, 0, 333, 2048, 1500, 64] * 5
    B, width = len(lengths), 5008 // page
    n_pages, guard = B * width, 1 << 20
    size = eora.cache_attention_workspace_bytes(B, heads, kv, dim, width * page)
    g = torch.Generator(device="cuda")
    g.manual_seed(dim)
    kind = torch.float16 if bits == 16 else torch.float8_e4m3fn
    k, v = (torch.randn((n_pages, kv, page, dim), generator=g, device="cuda", dtype=torch.float16).to(kind) for _ in range(2))
    scales = torch.ones(kv, device="cuda") if bits == 8 else None
    q = torch.randn((B, heads, dim), generator=g, device="cuda").half()
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(B, width)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = []
    for fill in (0, 255):
        buffer = torch.full((size + guard,), fill, dtype=torch.uint8, device="cuda")
        buffer[:HEAD] = 0
        buffer[size:] = 123
        for _ in range(3):
            out, lse = torch.empty((B, heads, dim), dtype=torch.float16, device="cuda"), torch.empty((B, heads), device="cuda")
            eora.cache_attention(q, k, v, scales, scales, table, n, out, lse, B, heads, kv, dim, heads * dim, n_pages, page, bits, width, 0, dim ** -0.5, buffer[:size])
            got.append((out, lse))
        torch.cuda.synchronize()
        assert bool((buffer[size:] == 123).all()) and not buffer[:HEAD].any()
    assert torch.isfinite(got[0][0]).all()
    assert all(torch.equal(o, got[0][0]) and torch.equal(s, got[0][1]) for o, s in got)
