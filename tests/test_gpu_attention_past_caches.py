"""eora_cache_attention where the requests hold so much that keys and values are read past the caches (112 MiB and more), against 64 bits on the GPU, and with
little in a table as wide: requests without a token, of one, ending inside tiles, with holes in their tables and NaN in every place that is not theirs.

Tolerance, element by element (u = 2^-11; L: largest sum of |scale q k| of a row): u |out| + 2^-17 (1 + L) sum p |v| + 2^-25: one rounding of the result; a weight's error of 2^-19 (1 + L),
once in the sum over v and once in the sum of weights, and fp32 sums in chains of at most some 100 additions.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2410_21271_amd as eora
    return eora


@pytest.mark.parametrize("much", [True, False])
@pytest.mark.parametrize("heads,kv,dim,bits,page,window", [
    (8, 2, 64, 16, 16, 0), (13, 13, 64, 8, 48, 0), (32, 8, 128, 16, 16, 0), (12, 4, 128, 8, 64, 7000), (4, 2, 256, 16, 32, 0), (17, 1, 256, 8, 80, 0),
])
def test_much_and_little(gpu, heads, kv, dim, bits, page, window, much):
    import torch
    rng = np.random.default_rng(dim + heads + bits)
    token = kv * dim * (bits // 8) * 2
    total = (120 << 20) // token if much else 3000
    B = 24
    share = rng.uniform(0.3, 1.7, B)
    lengths = (share / share.sum() * total * (1.6 if window else 1.1)).astype(int) | 1
    lengths[[3, 7, 11]] = [0, 1, 33]
    lengths[5] += max(0, total + 1000 - lengths.sum())
    assert not window or not much or np.minimum(lengths, window).sum() * token >= 112 << 20
    used = -(-lengths // page)
    width = max(int(used.max()), -(-((116 << 20) // token) // (B * page)) + 1 if not window else 0)
    n_pages = int(used.sum()) + 2
    g = torch.Generator(device="cuda")
    g.manual_seed(dim + bits)
    kind = torch.float16 if bits == 16 else torch.float8_e4m3fn
    k, v = (torch.randn((n_pages, kv, page, dim), generator=g, device="cuda", dtype=torch.float16).to(kind) for _ in range(2))
    order, table = rng.permutation(n_pages), np.full((B, width), -1, np.int32)
    mine = np.zeros((n_pages, page), bool)
    holes = np.zeros((B, width), bool)
    at = 0
    for b in range(B):
        for p in range(used[b]):
            table[b, p] = order[at]
            mine[order[at], :min(page, lengths[b] - p * page)] = True
            at += 1
        if used[b] > 4:
            holes[b, 2] = True
            mine[table[b, 2]] = False
            table[b, 2] = n_pages + 5
    none = torch.from_numpy(~mine).cuda()[:, None, :, None]
    for t in (k, v):                         # NaN: 0x7E00, 0x7F
        raw = t.view(torch.int16 if bits == 16 else torch.uint8)
        raw.masked_fill_(none, 0x7E00 if bits == 16 else 0x7F)
    ks, vs = (torch.rand(kv, generator=g, device="cuda") + 0.5 for _ in range(2)) if bits == 8 else (None, None)
    q = (0.5 * torch.randn((B, heads, dim), generator=g, device="cuda")).half()
    dev_table, dev_lengths = torch.from_numpy(table).cuda(), torch.from_numpy(lengths.astype(np.int32)).cuda()
    out, lse = torch.full((B, heads, dim), 7.0, device="cuda").half(), torch.zeros((B, heads), device="cuda")
    scale = dim ** -0.5
    gpu.cache_attention(q, k, v, ks, vs, dev_table, dev_lengths, out, lse, B, heads, kv, dim, heads * dim, n_pages, page, bits, width, window, scale,
                        gpu.new_attention_workspace(B, heads, kv, dim, width * page))
    torch.cuda.synchronize()
    group = heads // kv
    for b in range(B):
        n = int(lengths[b])
        t = np.arange(max(0, n - window) if window else 0, n)
        t = t[~holes[b, t // page]]
        if len(t) == 0:
            assert not out[b].any() and bool((lse[b] == -np.inf).all())
            continue
        pages, place = torch.from_numpy(table[b, t // page].astype(np.int64)).cuda(), torch.from_numpy(t % page).cuda()
        for h in range(kv):
            K, V = (x.view(torch.int16 if bits == 16 else torch.uint8)[pages, h, place].contiguous().view(kind).double() for x in (k, v))
            if bits == 8:
                K, V = K * ks[h].double(), V * vs[h].double()
            Q = q[b, h * group:(h + 1) * group].double()
            s = scale * (Q @ K.t().contiguous())
            p = torch.softmax(s, -1)
            want, size, L = p @ V, p @ V.abs(), (scale * (Q.abs() @ K.abs().t().contiguous())).amax(-1, keepdim=True)
            got = out[b, h * group:(h + 1) * group].double()
            off = (got - want).abs() - (2.0 ** -11 * want.abs() + 2.0 ** -17 * (1 + L) * size + 2.0 ** -25)
            assert bool((off <= 0).all()), "request %d of %d tokens, head %d: %d off" % (b, n, h, int((~(off <= 0)).sum()))
            gap = (lse[b, h * group:(h + 1) * group].double() - torch.logsumexp(s, -1)).abs()
            assert bool((gap <= 2.0 ** -17 * (1 + L[:, 0])).all())
