"""eora_cache_attention gives equal bits, in out and in lse, whoever is the last to arrive: calls whose units have parts from whole workgroups and from single
wavefronts, more of them than are joined at a time, many times over."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


def several(seed, n, lo, hi):
    import random
    rng = random.Random(seed)
    return [int(lo * (hi / lo) ** rng.random()) for _ in range(n)]


@pytest.mark.parametrize("lengths,heads,kv,dim,bits,page,window", [
    ([9000, 3, 0, 1], 4, 1, 128, 8, 16, 0),
    (several(1, 37, 1, 3001), 13, 13, 64, 16, 48, 1000),
    (several(2, 37, 200, 3001), 13, 13, 64, 8, 48, 1000),
    (several(3, 64, 1, 4096), 32, 8, 128, 16, 16, 0),
    (several(4, 23, 30, 2000), 12, 3, 256, 16, 32, 0),
    (several(5, 300, 1, 900), 8, 2, 64, 8, 16, 0),
])
def test_equal_bits_every_time(gpu, lengths, heads, kv, dim, bits, page, window):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(len(lengths) + dim)
    B, width = len(lengths), -(-max(lengths) // page)
    n_pages = B * width
    kind = torch.float16 if bits == 16 else torch.float8_e4m3fn
    k, v = (torch.randn((n_pages, kv, page, dim), generator=g, device="cuda", dtype=torch.float16).to(kind) for _ in range(2))
    scales = torch.full((kv,), 0.9, device="cuda") if bits == 8 else None
    q = torch.randn((B, heads, dim), generator=g, device="cuda").half()
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(B, width)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ws = gpu.new_attention_workspace(B, heads, kv, dim, width * page)

    def run():
        out, lse = torch.empty((B, heads, dim), dtype=torch.float16, device="cuda"), torch.empty((B, heads), device="cuda")
        gpu.cache_attention(q, k, v, scales, scales, table, n, out, lse, B, heads, kv, dim, heads * dim, n_pages, page, bits, width, window, dim ** -0.5, ws)
        return out, lse

    out, lse = run()
    assert torch.isfinite(out).all()
    other = torch.zeros((), dtype=torch.int64, device="cuda")
    for i in range(400):
        again = run()
        other += (again[0].view(torch.int16) != out.view(torch.int16)).sum() + (again[1].view(torch.int32) != lse.view(torch.int32)).sum()
        if i % 4 == 3:
            k.view(torch.int8)[i % n_pages].add_(0)       # (what the caches hold changes from call to call)
    assert int(other) == 0, "%d values with other bits in 400 calls" % int(other)
