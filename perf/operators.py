"""The operators between the linears of a decoder layer, as cases that can be timed and compared.

A serving step over compressed linears is: the query / key / value projections, the requests' own low-rank pairs beside
them ("adapters"), the norms and position rotations of query and key heads with the new keys and values stored in a paged
cache ("append"), and the attention of the new tokens over that cache ("attention").

    adapters   y[m] = base[m] + s_a (x[m] A_a^T) B_a^T, a = adapter_of_row[m], pairs from a pool
    append     per head: n = x rsqrt(mean x^2 + eps) w; pairs of columns rotated by the token's position; k and v to their slots
    attention  out = softmax(scale q K^T) V over the pages of each request

Inputs are synthetic: LLaMA-3-shaped layers and odd sizes, Gaussian activations with outlier channels, factors and caches.
"""
import math
import random

import torch

own = False

HEADS_8B = dict(heads=32, kv=8, dim=128)
HEADS_70B = dict(heads=64, kv=8, dim=128)
EPS = 1e-5
POSITIONS = 1 << 17                                       # rows of the table of rotations (a 128 Ki context)


def listed():
    return [
        # one request with a pair of its own beside one small projection: launches and host time count
        dict(name="adapters, 1 token", kind="adapters", M=1, d_in=1024, d_out=1024, r=64, n=4, bits=16, rows="random", mixed=False, pattern=1),
        # a serving batch beside the 8B query projection, 256 pairs loaded, ranks 32 to 128 mixed, a few requests without one
        dict(name="adapters 8B, 64 requests", kind="adapters", M=64, d_in=4096, d_out=4096, r=128, n=256, bits=16, rows="random", mixed=True, pattern=2),
        # sizes that are no powers of two, 4-bit pairs, several requests to a pair
        dict(name="adapters ragged q4, 37 req.", kind="adapters", M=37, d_in=2688, d_out=7296, r=256, n=20, bits=4, rows="random", mixed=True, pattern=3),
        # prompts of several requests in one batch, beside the 8B gate projection
        dict(name="adapters 8B, 2048 tokens", kind="adapters", M=2048, d_in=4096, d_out=14336, r=128, n=8, bits=16, rows="runs", mixed=False, pattern=4),
        # one new token of an 8B model
        dict(name="append 8B, 1 token", kind="append", M=1, bits=16, page=16, norm=False, rot=128, interleaved=False, **HEADS_8B),
        # prompts of odd length, few and narrow heads, half of each head rotated, pages that are no power of two
        dict(name="append ragged, 1777 tokens", kind="append", M=1777, heads=12, kv=3, dim=64, bits=16, page=48, norm=True, rot=32, interleaved=True),
        # a long prompt of a 70B model into an 8-bit cache, with norms
        dict(name="append 70B q8, 8192 tokens", kind="append", M=8192, bits=8, page=64, norm=True, rot=128, interleaved=False, **HEADS_70B),
        # one request that has just begun
        dict(name="attention 8B, 1 x 100", kind="attention", B=1, longest=100, shortest=100, bits=16, page=16, window=0, pattern=1, **HEADS_8B),
        # a serving batch of an 8B model, short and long requests together
        dict(name="attention 8B, 64 x 1..4096", kind="attention", B=64, longest=4096, shortest=1, bits=16, page=16, window=0, pattern=2, **HEADS_8B),
        # one key-value head per query head, narrow heads, odd numbers of everything, the last 1000 tokens only
        dict(name="attention ragged, 37 req.", kind="attention", B=37, longest=3001, shortest=0, heads=13, kv=13, dim=64, bits=16, page=48, window=1000, pattern=3),
        # one request with a long document, 70B heads, 8-bit cache
        dict(name="attention 70B q8, 1 x 131072", kind="attention", B=1, longest=131072, shortest=131072, bits=8, page=64, window=0, pattern=4, **HEADS_70B),
        # a full serving batch of a 70B model, 8-bit cache
        dict(name="attention 70B q8, 160 x 8192", kind="attention", B=160, longest=8192, shortest=1024, bits=8, page=64, window=0, pattern=5, **HEADS_70B),
    ]


def _log(rng, lo, hi):
    """A whole number, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the same ranges: any shape the entry points take, odd ones among them."""
    kind = rng.choice(("adapters", "append", "attention", "attention"))
    pattern = rng.randrange(1 << 20)
    if kind == "adapters":
        bits = rng.choice((16, 16, 4, 3))
        r = 32 * _log(rng, 1, 8) if bits == 16 else (rng.choice((64, 128, 256)) if bits == 4 else rng.choice((128, 256)))
        M = _log(rng, 1, 2048)
        d_in, d_out = 128 * _log(rng, 4, 64), 16 * _log(rng, 16, 896)
        n = _log(rng, 1, 256) if M <= 256 else _log(rng, 1, 8)
        return dict(kind=kind, M=M, d_in=d_in, d_out=d_out, r=r, n=n, bits=bits, rows="random" if M <= 256 else "runs", mixed=rng.random() < 0.6, pattern=pattern)
    dim = rng.choice((64, 128, 128, 256))
    kv = rng.choice((1, 2, 3, 5, 8, 8, 12))
    heads = kv * rng.choice((1, 2, 4, 4, 5, 8))
    bits, page = rng.choice((16, 8)), 16 * _log(rng, 1, 16)
    if kind == "append":
        rot = rng.choice((dim, dim, dim // 2, 16 * rng.randint(0, dim // 16)))
        return dict(kind=kind, M=_log(rng, 1, min(8192, 8192 * 10240 // ((heads + 2 * kv) * dim))), heads=heads, kv=kv, dim=dim, bits=bits, page=page,
                    norm=rng.random() < 0.5, rot=rot, interleaved=rng.random() < 0.3)
    B = _log(rng, 1, 160)
    longest = _log(rng, 1, min(131072, 160 * 8192 * 8 * 128 // (2 * B * kv * dim)))
    shortest = rng.choice((0, 1, max(1, longest // 8), longest))
    return dict(kind=kind, B=B, longest=longest, shortest=shortest, heads=heads, kv=kv, dim=dim, bits=bits, page=page,
                window=rng.choice((0, 0, 0, _log(rng, 1, longest))), pattern=pattern)


# ---------------------------------------------------------------------------------------------------- what a case says
def _step(case):
    """Ranks come in whole tiles of the stored B."""
    return 32 if case["bits"] == 16 else min(128, case["r"])


def _rows_of(case):
    """(adapter of each row, rank of each adapter)."""
    rng = random.Random(case["pattern"])
    M, n, step = case["M"], case["n"], _step(case)
    ranks = [step * rng.randint(1, case["r"] // step) if case["mixed"] else case["r"] for _ in range(n)]
    if case["rows"] == "random":                          # one new token of each request, some without a pair
        return [rng.randint(-1, n - 1) if M > 1 else rng.randrange(n) for _ in range(M)], ranks
    cuts = sorted(rng.randrange(M) for _ in range(n - 1))       # prompts one after the other
    ids = [rng.randrange(n) if rng.random() < 0.9 else -1 for _ in range(n)]
    return [ids[sum(c <= m for c in cuts)] for m in range(M)], ranks


def _lengths_of(case):
    rng = random.Random(case["pattern"])
    lo, hi = case["shortest"], case["longest"]
    got = [lo if lo == hi else min(hi, (_log(rng, max(1, lo), hi) if rng.random() < 0.95 else lo)) for _ in range(case["B"])]
    got[rng.randrange(case["B"])] = hi
    return got


def _factor_bytes(case, rank):
    """Stored bytes of one pair of a rank."""
    d, bits = case["d_in"] + case["d_out"], case["bits"]
    if bits == 16:
        return 2 * rank * d
    return rank * d * bits / 8 + 2 * rank * (case["d_in"] // 128) + 2 * case["d_out"] * (rank // _step(case))


def work(case):
    if case["kind"] == "adapters":
        ids, ranks = _rows_of(case)
        M, d_in, d_out = case["M"], case["d_in"], case["d_out"]
        used = {a for a in ids if a >= 0}
        return {"bytes": 2 * M * d_in + 4 * M * d_out + 4 * M + sum(_factor_bytes(case, ranks[a]) + 8 for a in used),
                "flops": sum(2 * ranks[a] * (d_in + d_out) for a in ids if a >= 0)}
    heads, kv, dim, size = case["heads"], case["kv"], case["dim"], case["bits"] // 8
    if case["kind"] == "append":
        M = case["M"]
        return {"bytes": M * (2 * (2 * heads + 2 * kv) * dim + 2 * kv * dim * size + 4 * case["rot"] + 12),
                "flops": M * (heads + kv) * (4 * dim * bool(case["norm"]) + 3 * case["rot"])}
    lens = _lengths_of(case)
    total = sum(min(n, case["window"]) if case["window"] else n for n in lens)
    return {"bytes": total * 2 * kv * dim * size + 4 * case["B"] * heads * dim + 4 * case["B"] * (1 + heads) + 4 * total // case["page"],
            "flops": 4 * total * heads * dim}


# ---------------------------------------------------------------------------------------------------- what a program has in hand
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float16, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _words(g, rows, cols, bits):
    """Stored 4- or 3-bit codes of a symmetric quantiser, in whatever order: all of them are drawn alike."""
    zero = 1 << (bits - 1)

    def codes(*shape):
        return (torch.randn(shape, generator=g, device="cuda") * (zero / 2.5) + zero).round_().clamp_(1, 2 * zero - 1).to(torch.int32)

    if bits == 4:
        return (codes(rows * cols // 8, 8) << (4 * torch.arange(8, device="cuda", dtype=torch.int32))).sum(-1, dtype=torch.int64).to(torch.int32)
    c = codes(rows * cols // 32, 3, 10).to(torch.int64)
    low = (c[..., :5] << (3 * torch.arange(5, device="cuda"))).sum(-1) + (c[..., 5:] << (16 + 3 * torch.arange(5, device="cuda"))).sum(-1)
    last = codes(rows * cols // 32, 2).to(torch.int64)
    bit = torch.arange(3, device="cuda")
    low = low + (((last[:, :1] >> bit) & 1) << 15) + (((last[:, 1:] >> bit) & 1) << 31)
    return torch.where(low >= 1 << 31, low - (1 << 32), low).to(torch.int32).reshape(-1)


def _rotations(rot):
    """(cos, sin) of the positions times the usual frequencies, in fp32."""
    if rot == 0:
        return None
    f = 500000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
    a = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["kind"] == "adapters":
        M, d_in, d_out, r, n, bits = (case[k] for k in ("M", "d_in", "d_out", "r", "n", "bits"))
        ids, ranks = _rows_of(case)
        x = torch.randn((M, d_in), generator=g, device="cuda")
        x[:, torch.randperm(d_in, generator=g, device="cuda")[: max(1, d_in // 100)]] *= 8.0      # outlier channels
        s.update(x=x.half(), base=_randn(g, M, d_out), y=torch.empty((M, d_out), device="cuda", dtype=torch.float16),
                 ids=torch.tensor(ids, dtype=torch.int32, device="cuda"), ranks=torch.tensor(ranks, dtype=torch.int32, device="cuda"),
                 scalings=torch.rand(n, generator=g, device="cuda") + 0.5)
        if bits == 16:
            s.update(A=_randn(g, n, r * d_in, scale=d_in ** -0.5), B=_randn(g, n, d_out * r, scale=0.5 * r ** -0.5), As=None, Bs=None)
        else:
            top = (1 << (bits - 1)) / 2.5                 # code steps to a standard deviation
            s.update(A=torch.stack([_words(g, r, d_in, bits) for _ in range(n)]), B=torch.stack([_words(g, d_out, r, bits) for _ in range(n)]),
                     As=((torch.rand((n, r, d_in // 128), generator=g, device="cuda") + 0.5) * d_in ** -0.5 / top).half(),
                     Bs=((torch.rand((n, d_out, r // min(128, r)), generator=g, device="cuda") + 0.5) * 0.5 * r ** -0.5 / top).half())
        return s
    heads, kv, dim, bits, page = (case[k] for k in ("heads", "kv", "dim", "bits", "page"))
    if bits == 8:
        s.update(k_scale=(torch.rand(kv, generator=g, device="cuda") + 0.5) * 0.01, v_scale=(torch.rand(kv, generator=g, device="cuda") + 0.5) * 0.01)
    else:
        s.update(k_scale=None, v_scale=None)
    if case["kind"] == "append":
        M = case["M"]
        pages = -(-M // page) + 2
        s.update(q=_randn(g, M, heads, dim), k=_randn(g, M, kv, dim), v=_randn(g, M, kv, dim), q_out=torch.empty((M, heads, dim), device="cuda", dtype=torch.float16),
                 q_weight=_randn(g, dim, scale=0.2) + 1 if case["norm"] else None, k_weight=_randn(g, dim, scale=0.2) + 1 if case["norm"] else None,
                 rotations=_rotations(case["rot"]), rot=case["rot"], interleaved=case["interleaved"])
        # the tokens of one prompt, from some position on, into pages in any order; one row in a hundred is padding
        first = torch.randint(0, POSITIONS - M, (1,), generator=g, device="cuda")
        at = torch.arange(M, device="cuda")
        slots = torch.randperm(pages, generator=g, device="cuda")[at // page] * page + at % page
        s.update(positions=(first + at).to(torch.int32), slots=torch.where(at % 100 == 99, -1, slots))
        s.update(pages_k=torch.zeros((pages, kv, page, dim), device="cuda", dtype=torch.float16), pages_v=torch.zeros((pages, kv, page, dim), device="cuda", dtype=torch.float16))
        if bits == 8:
            s.update(pages_k=s["pages_k"].to(torch.float8_e4m3fn), pages_v=s["pages_v"].to(torch.float8_e4m3fn))
        return s
    lens, B = _lengths_of(case), case["B"]
    width = max(1, -(-case["longest"] // page))
    used = [-(-n // page) for n in lens]
    pages = sum(used) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    ends = torch.tensor(used, device="cuda").cumsum(0)
    col = torch.arange(width, device="cuda")[None]
    at = (ends - torch.tensor(used, device="cuda"))[:, None] + col
    table = torch.where(col < torch.tensor(used, device="cuda")[:, None], order[at.clamp(max=pages - 1)], -1).to(torch.int32)
    s.update(q=_randn(g, B, heads, dim, scale=1.5), table=table, lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             out=torch.empty((B, heads, dim), device="cuda", dtype=torch.float16), lse=torch.empty((B, heads), device="cuda", dtype=torch.float32))
    for name, scale in (("pages_k", s["k_scale"]), ("pages_v", s["v_scale"])):
        t = torch.randn((pages, kv, page, dim), generator=g, device="cuda", dtype=torch.float16)
        s[name] = t if bits == 16 else (t * (1.0 / scale).half()[:, None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"adapters": _adapters, "append": _append, "attention": _attention}[s["case"]["kind"]](s)


def _plain_factor(t, scales, rows, cols, bits):
    """Stored tiles of some pairs (pair x words) -> pair x rows x cols in fp32."""
    u = t.shape[0]
    if bits == 16:                                        # 16 x 32 tiles; lane 16 j + n: columns 8 j .. 8 j + 7 of row n
        return t.view(u, rows // 16, cols // 32, 4, 16, 8).permute(0, 1, 4, 2, 3, 5).reshape(u, rows, cols).float()
    wide = min(128, cols)
    col = torch.arange(wide // 4, device=t.device)        # a lane's columns
    if bits == 4:                                         # word c / 8, nibble 4 (c % 2) + (c % 8) / 2
        w = t.view(u, rows // 16, cols // wide, 4, 16, wide // 32)
        code = (w[..., col // 8] >> (4 * (4 * (col % 2) + col % 8 // 2)).to(torch.int32)) & 15
    else:                                                 # pair p < 15: word p / 5 at 16 h + 3 (p % 5); the last one in bits 15 and 31
        w = t.view(u, rows // 16, cols // wide, 4, 16, 3)
        p, h = (col // 2)[:30], (col % 2)[:30]
        code = (w[..., p // 5] >> (16 * h + 3 * (p % 5)).to(torch.int32)) & 7
        bit = torch.arange(3, device=t.device, dtype=torch.int32)
        last = torch.stack([(((w >> at) & 1) << bit).sum(-1, dtype=torch.int32) for at in (15, 31)], -1)
        code = torch.cat((code, last), -1)
    code = code.permute(0, 1, 4, 2, 3, 5).reshape(u, rows, cols // wide, wide)
    return ((code - (1 << (bits - 1))).float() * scales.view(u, rows, cols // wide, 1).float()).reshape(u, rows, cols)


def _adapters(s):
    c = s["case"]
    M, d_in, d_out, r, n, bits = (c[k] for k in ("M", "d_in", "d_out", "r", "n", "bits"))
    if own:
        import paper_2410_21271_amd as eora
        if "workspace" not in s:
            s["workspace"] = eora.new_adapters_workspace(M, d_in, d_out, r)
        eora.linear_adapters(s["x"], s["A"], s["B"], s["As"], s["Bs"], s["ranks"], s["scalings"], s["ids"], s["base"], s["y"],
                             M, d_in, d_out, r, n, bits, s["workspace"])
        return s["y"]
    ids = s["ids"].long()
    used, which = torch.unique(ids.clamp(min=0), return_inverse=True)
    pick = lambda t: None if t is None else t[used]       # noqa: E731
    A = _plain_factor(pick(s["A"]), pick(s["As"]), r, d_in, bits)
    B = _plain_factor(pick(s["B"]), pick(s["Bs"]), d_out, r, bits)
    t = (s["x"].float() @ A.reshape(-1, d_in).t()).view(M, -1, r)
    mine = (which[:, None] == torch.arange(len(used), device=ids.device)) & (ids >= 0)[:, None]
    keep = mine[:, :, None] & (torch.arange(r, device=ids.device) < s["ranks"][used][:, None])[None]
    t = torch.where(keep, t * s["scalings"][used][:, None], 0.0)
    return (s["base"].float() + t.view(M, -1) @ B.transpose(1, 2).reshape(-1, d_out)).half()


def _plain_heads(x, weight, cs, rot, interleaved):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    if rot == 0:
        return x
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., : rot // 2], head[..., rot // 2:])
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1), rest), -1)


def _append(s):
    c = s["case"]
    heads, kv, dim, bits, page, rot = (c[k] for k in ("heads", "kv", "dim", "bits", "page", "rot"))
    if own:
        import paper_2410_21271_amd as eora
        eora.cache_append(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["rotations"], s["positions"], s["slots"], s["q_out"],
                          s["pages_k"], s["pages_v"], s["k_scale"], s["v_scale"], c["M"], heads, kv, dim, heads * dim, kv * dim, kv * dim,
                          rot, c["interleaved"], POSITIONS if rot else 0, EPS, s["pages_k"].shape[0], page, bits)
        return {"q": s["q_out"], "k": s["pages_k"], "v": s["pages_v"]}
    cs = s["rotations"][s["positions"].long()] if rot else None
    q = _plain_heads(s["q"], s["q_weight"], cs, rot, c["interleaved"])
    k = _plain_heads(s["k"], s["k_weight"], cs, rot, c["interleaved"])
    v = s["v"].float()
    live = s["slots"] >= 0
    slot = s["slots"][live]
    if bits == 8:
        k, v = ((t / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for t, scale in ((k, s["k_scale"]), (v, s["v_scale"])))
    else:
        k, v = k.half(), v.half()
    s["pages_k"].view(k.dtype)[slot // page, :, slot % page] = k[live]
    s["pages_v"].view(v.dtype)[slot // page, :, slot % page] = v[live]
    return {"q": q.half(), "k": s["pages_k"], "v": s["pages_v"]}


def _attention(s):
    c = s["case"]
    B, heads, kv, dim, bits, page, window = (c[k] for k in ("B", "heads", "kv", "dim", "bits", "page", "window"))
    width, scale = s["table"].shape[1], dim ** -0.5
    if own:
        import paper_2410_21271_amd as eora
        if "workspace" not in s:
            s["workspace"] = eora.new_attention_workspace(B, heads, kv, dim, width * page)
        eora.cache_attention(s["q"], s["pages_k"], s["pages_v"], s["k_scale"], s["v_scale"], s["table"], s["lengths"], s["out"], s["lse"],
                             B, heads, kv, dim, heads * dim, s["pages_k"].shape[0], page, bits, width, window, scale, s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    at = s["table"].clamp(min=0).long()

    def rows(pages, by):
        t = pages.view(torch.uint8)[at].view(pages.dtype).float() if bits == 8 else pages[at].float()
        t = t.permute(0, 2, 1, 3, 4).reshape(B, kv, width * page, dim)
        return t if by is None else t * by[:, None, None]

    n, pos = s["lengths"].long()[:, None], torch.arange(width * page, device=at.device)
    keep = ((pos < n) & (pos >= (n - window if window else 0)) & (s["table"] >= 0).repeat_interleave(page, 1))[:, None, None]
    score = torch.matmul(s["q"].float().view(B, kv, heads // kv, dim), rows(s["pages_k"], s["k_scale"]).transpose(-1, -2)) * scale
    score = torch.where(keep, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, rows(s["pages_v"], s["v_scale"])) / torch.where(total == 0, 1.0, total)
    return {"out": out.half().view(B, heads, dim), "lse": (top + torch.log(total)).view(B, heads)}


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_factor(t, scales, rows, cols, bits):
    """One pair's stored tiles, element by element: where row i, column c lies."""
    i, c = torch.meshgrid(torch.arange(rows, device="cuda"), torch.arange(cols, device="cuda"), indexing="ij")
    if bits == 16:
        return t[((i // 16) * (cols // 32) + c // 32) * 512 + (16 * (c % 32 // 8) + i % 16) * 8 + c % 8].double()
    wide = min(128, cols)
    per = wide * bits // 128                              # words of a lane
    tile, lane, at = (i // 16) * (cols // wide) + c // wide, 16 * (c % wide // (wide // 4)) + i % 16, c % (wide // 4)
    word = lambda w: t[(tile * 64 + lane) * per + w].long() & 0xFFFFFFFF       # noqa: E731
    if bits == 4:
        code = (word(at // 8) >> (16 * (at % 2) + 4 * (at % 8 // 2))) & 15
    else:
        spread = sum(((word(b) >> (15 + 16 * (at % 2))) & 1) << b for b in range(3))
        code = torch.where(at < 30, (word((at // 2).clamp(max=14) // 5) >> (16 * (at % 2) + 3 * (at // 2 % 5))) & 7, spread)
    return (code - (1 << (bits - 1))).double() * scales.double().reshape(rows, cols // wide).repeat_interleave(wide, 1)


def _exact_adapters(c, s):
    y = s["base"].double()
    ids, ranks = _rows_of(c)
    for a in sorted({i for i in ids if i >= 0}):
        rows = torch.tensor([m for m, i in enumerate(ids) if i == a], device="cuda")
        scales = (None, None) if c["bits"] == 16 else (s["As"][a], s["Bs"][a])
        A = _exact_factor(s["A"][a], scales[0], c["r"], c["d_in"], c["bits"])[: ranks[a]]
        B = _exact_factor(s["B"][a], scales[1], c["d_out"], c["r"], c["bits"])[:, : ranks[a]]
        y[rows] += s["scalings"][a].double() * ((s["x"][rows].double() @ A.t().contiguous()) @ B.t().contiguous())
    return y


def _exact_append(c, s):
    rot, dim, page = c["rot"], c["dim"], c["page"]

    def turned(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / dim + EPS) * weight.double()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
            cs = s["rotations"][s["positions"].long(), i].double()
            z = torch.complex(x[..., a], x[..., b]) * torch.complex(cs[:, :1], cs[:, 1:])
            x[..., a], x[..., b] = z.real, z.imag
        return x

    got = {"q": turned(s["q"].clone(), s["q_weight"])}
    live = (s["slots"] >= 0).nonzero()[:, 0]
    slot = s["slots"][live]
    for name, rows, by in (("k", turned(s["k"].clone(), s["k_weight"]), s["k_scale"]), ("v", s["v"].double(), s["v_scale"])):
        pages = s["pages_" + name].double().transpose(1, 2).reshape(-1, c["kv"], dim).contiguous()
        pages[slot] = rows[live] if by is None else rows[live] / by.double()[:, None]
        got[name] = pages.view(-1, page, c["kv"], dim).transpose(1, 2).contiguous()
    return got


def _exact_attention(c, s):
    B, heads, kv, dim, page = (c[k] for k in ("B", "heads", "kv", "dim", "page"))
    out = torch.zeros((B, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((B, heads), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths_of(c)):
        if n == 0:
            continue
        at = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device="cuda")
        pages, place = s["table"][b].long()[at // page], at % page
        for h in range(kv):
            one = slice(h * (heads // kv), (h + 1) * (heads // kv))
            K, V = (s[t].view(torch.uint8)[pages, h, place].view(s[t].dtype) if c["bits"] == 8 else s[t][pages, h, place] for t in ("pages_k", "pages_v"))
            K, V = (t.double() * (1.0 if by is None else by[h].double()) for t, by in ((K, s["k_scale"]), (V, s["v_scale"])))
            score = (s["q"][b, one].double() @ K.t().contiguous()) / math.sqrt(dim)
            lse[b, one] = torch.logsumexp(score, -1)
            out[b, one] = torch.softmax(score, -1) @ V
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"adapters": _exact_adapters, "append": _exact_append, "attention": _exact_attention}[case["kind"]](case, s)
