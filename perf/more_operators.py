"""The paged cache with a scale for each block of tokens, and attention of single tokens and of prompts over it, as cases that can be timed and compared.

    blocks     new queries, keys and values (norm, rotation as of a decoder layer) stored as e4m3 codes with a power of two for each 16 tokens
               and head, which grows with the block's values; then the request's last blocks read back as fp16
    token      one new token per request:  out = softmax(scale q K^T) V over the last `window` tokens and the first `sinks`
    prompt     the last rows of each request at once, each of which sees the tokens up to its own, the last `window` of them and the first `sinks`

Inputs are synthetic: LLaMA-3-shaped layers and odd sizes, Gaussian activations and caches.
"""
import math
import random

import torch

own = False

HEADS_8B = dict(heads=32, kv=8, dim=128)
HEADS_70B = dict(heads=64, kv=8, dim=128)
EPS = 1e-5
POSITIONS = 1 << 17                                       # rows of the table of rotations (a 128 Ki context)
BLOCK = 16                                                # tokens that share a scale
LEAST, MOST = -15, 8                                      # powers of two: every code stands for an fp16 number
TOP = 448.0                                               # the largest e4m3 code


def listed():
    return [
        # one new token of an 8B model, into a block that others have begun
        dict(name="blocks 8B, 1 token", kind="blocks", M=1, requests=1, page=16, norm=False, rot=128, interleaved=False, pattern=1, **HEADS_8B),
        # pieces of several prompts, few and narrow heads, half of each head rotated, pages that are no power of two
        dict(name="blocks ragged, 1777 tokens", kind="blocks", M=1777, requests=9, heads=12, kv=3, dim=64, page=48, norm=True, rot=32, interleaved=True, pattern=2),
        # a long prompt of a 70B model, with norms
        dict(name="blocks 70B, 8192 tokens", kind="blocks", M=8192, requests=1, page=64, norm=True, rot=128, interleaved=False, pattern=3, **HEADS_70B),
        # one request that has just begun
        dict(name="token 8B, 1 x 100", kind="token", B=1, longest=100, shortest=100, cache="blocks", page=16, window=0, sinks=0, pattern=4, **HEADS_8B),
        # a serving batch of an 8B model that looks back at 2048 tokens and at how each request began
        dict(name="token 8B, 64 x 1..8192, window", kind="token", B=64, longest=8192, shortest=1, cache="blocks", page=16, window=2048, sinks=16, pattern=5, **HEADS_8B),
        # one key-value head per query head, narrow heads, odd numbers of everything
        dict(name="token ragged, 37 req., window", kind="token", B=37, longest=3001, shortest=0, heads=13, kv=13, dim=64, cache="fp16", page=48, window=1000, sinks=37, pattern=6),
        # a full serving batch of a 70B model
        dict(name="token 70B, 160 x 8192", kind="token", B=160, longest=8192, shortest=1024, cache="blocks", page=64, window=0, sinks=0, pattern=7, **HEADS_70B),
        # a short question
        dict(name="prompt 8B, 17 rows", kind="prompt", B=1, rows=17, even=True, longest=17, cache="fp16", page=16, window=0, sinks=0, pattern=8, **HEADS_8B),
        # a prompt of an 8B model
        dict(name="prompt 8B, 2048 rows", kind="prompt", B=1, rows=2048, even=True, longest=2048, cache="blocks", page=16, window=0, sinks=0, pattern=9, **HEADS_8B),
        # pieces of prompts and single tokens in one batch, five query heads to a key-value head, odd numbers of everything
        dict(name="prompt ragged, 11 req., window", kind="prompt", B=11, rows=500, even=False, longest=3001, heads=15, kv=3, dim=64, cache="fp16", page=48, window=1000, sinks=37, pattern=10),
        # five tokens of each request, drafted and to be looked at together
        dict(name="prompt 8B, 32 x 5 rows of 8192", kind="prompt", B=32, rows=5, even=True, longest=8192, cache="blocks", page=16, window=0, sinks=0, pattern=11, **HEADS_8B),
        # a long prompt of a 70B model
        dict(name="prompt 70B, 8192 rows", kind="prompt", B=1, rows=8192, even=True, longest=8192, cache="fp16", page=64, window=0, sinks=0, pattern=12, **HEADS_70B),
    ]


def _log(rng, lo, hi):
    """A whole number, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the same ranges: any shape the entry points take, odd ones among them."""
    kind = rng.choice(("blocks", "token", "prompt", "prompt"))
    pattern = rng.randrange(1 << 20)
    dim = rng.choice((64, 128, 128, 256))
    kv = rng.choice((1, 2, 3, 5, 8, 8, 12))
    heads = kv * rng.choice((1, 2, 4, 4, 5, 8))
    page = 16 * _log(rng, 1, 16)
    same = dict(kind=kind, heads=heads, kv=kv, dim=dim, page=page, pattern=pattern)
    if kind == "blocks":
        M = _log(rng, 1, min(8192, 8192 * 10240 // ((heads + 2 * kv) * dim)))
        return dict(M=M, requests=_log(rng, 1, min(M, 256)), norm=rng.random() < 0.5, rot=rng.choice((dim, dim, dim // 2, 16 * rng.randint(0, dim // 16))),
                    interleaved=rng.random() < 0.3, **same)
    cache = rng.choice(("fp16", "heads", "blocks", "blocks"))
    if kind == "token":
        B = _log(rng, 1, 160)
        longest = _log(rng, 1, min(131072, 160 * 8192 * 8 * 128 // (2 * B * kv * dim)))
        more = dict(B=B, longest=longest, shortest=rng.choice((0, 1, max(1, longest // 8), longest)))
    else:
        B = _log(rng, 1, 48)
        longest = _log(rng, 1, 8192)
        most = 64 * 8192 * 8192 * 128 // (2 * B * heads * dim * longest)      # rows that cost what the largest case does
        more = dict(B=B, longest=longest, rows=_log(rng, 1, max(1, min(longest, most))), even=rng.random() < 0.4)
    return dict(cache=cache, window=rng.choice((0, 0, _log(rng, 1, longest))), sinks=rng.choice((0, 1, 4, _log(rng, 1, 64))), **more, **same)


# ---------------------------------------------------------------------------------------------------- what a case says
def _spans_of(case):
    """(first new position, new tokens) of each request whose tokens are stored."""
    rng = random.Random(case["pattern"])
    M, n = case["M"], case["requests"]
    cuts = [0] + sorted(rng.sample(range(1, M), n - 1)) + [M] if n > 1 else [0, M]
    return [(rng.choice((0, rng.randrange(1, 4096))) if M > n else rng.randrange(1, 4096), b - a) for a, b in zip(cuts, cuts[1:])]


def _lengths_of(case):
    """(tokens, rows) of each request."""
    rng = random.Random(case["pattern"])
    B, hi = case["B"], case["longest"]
    if case["kind"] == "token":
        lo = case["shortest"]
        got = [lo if lo == hi else min(hi, (_log(rng, max(1, lo), hi) if rng.random() < 0.95 else lo)) for _ in range(B)]
        got[rng.randrange(B)] = hi
        return [(n, 1) for n in got]
    rows = [case["rows"] if case["even"] else _log(rng, 1, case["rows"]) for _ in range(B)]
    rows[rng.randrange(B)] = case["rows"]
    return [(hi if case["even"] else _log(rng, n, hi), n) for n in rows]


def _seen(case, tokens, rows):
    """(pairs of a row and a token that it sees, tokens that some row sees) of a request."""
    window, sinks = case["window"], case["sinks"]
    pairs, low = 0, None
    if window == 0:
        n = min(rows, tokens)
        return n * tokens - n * (n - 1) // 2, tokens if n else 0
    for p in range(max(0, tokens - rows), tokens):
        lo = max(0, p + 1 - window)
        low = lo if low is None else low
        pairs += p + 1 - lo + min(sinks, lo)
    return pairs, 0 if low is None else tokens - low + min(sinks, low)


def work(case):
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["kind"] == "blocks":
        M = case["M"]
        back = sum(at % BLOCK + n for at, n in _spans_of(case))
        return {"bytes": M * (2 * (2 * heads + 2 * kv) * dim + 2 * kv * dim + 4 * case["rot"] + 12) + back * (6 * kv * dim + 8),
                "flops": M * (heads + kv) * (4 * dim * bool(case["norm"]) + 3 * case["rot"]) + 2 * M * kv * dim}
    size = 2 if case["cache"] == "fp16" else 1
    got = [_seen(case, *r) for r in _lengths_of(case)]
    M, total = sum(n for _, n in _lengths_of(case)), sum(n for _, n in got)
    return {"bytes": total * 2 * kv * dim * size + 4 * M * heads * dim + 4 * M * heads + 8 * case["B"] + 4 * total // case["page"],
            "flops": 4 * sum(n for n, _ in got) * heads * dim}


# ---------------------------------------------------------------------------------------------------- what a program has in hand
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).half()


def _rotations(rot):
    """(cos, sin) of the positions times the usual frequencies, in fp32."""
    if rot == 0:
        return None
    f = 500000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
    a = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _stored(g, pages, kv, page, dim):
    """A cache of Gaussian values, as blocks have them: codes (pages x kv x page x dim) and bytes of the powers (pages x kv x page / 16)."""
    t = torch.randn((pages, kv, page // BLOCK, BLOCK, dim), generator=g, device="cuda", dtype=torch.float16)
    t *= (torch.rand((pages, kv, page // BLOCK, 1, 1), generator=g, device="cuda") * 1.5 + 0.5).half()
    e = torch.ceil(torch.log2(t.abs().amax((-1, -2)).float() / TOP)).clamp_(LEAST, MOST)
    t *= torch.exp2(-e).half()[..., None, None]
    return t.clamp_(-TOP, TOP).to(torch.float8_e4m3fn).view(pages, kv, page, dim), (e + 127).to(torch.uint8)


def _table(g, used, width):
    """Pages of each request, drawn without order: B x width, -1 behind the last."""
    pages = sum(used) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    n = torch.tensor(used, device="cuda")
    col = torch.arange(width, device="cuda")[None]
    at = (n.cumsum(0) - n)[:, None] + col
    return torch.where(col < n[:, None], order[at.clamp(max=pages - 1)], -1).to(torch.int32), pages


def prepare(case, seed):
    g = _gen(seed)
    heads, kv, dim, page = (case[k] for k in ("heads", "kv", "dim", "page"))
    s = {"case": case}
    if case["kind"] == "blocks":
        M, spans = case["M"], _spans_of(case)
        # a request's pages from the block on in which its new tokens begin: what lies before is not touched
        first = [at % page // BLOCK * BLOCK + at % BLOCK for at, _ in spans]
        used = [-(-(f + n) // page) for f, (_, n) in zip(first, spans)]
        table, pages = _table(g, used, max(used))
        who = torch.repeat_interleave(torch.arange(len(spans), device="cuda"), torch.tensor([n for _, n in spans], device="cuda"))
        begin = torch.tensor([n for _, n in spans], device="cuda").cumsum(0) - torch.tensor([n for _, n in spans], device="cuda")
        at = torch.arange(M, device="cuda") - begin[who]
        place = torch.tensor(first, device="cuda")[who] + at
        slots = table[who, place // page].long() * page + place % page
        back_who = torch.repeat_interleave(torch.arange(len(spans), device="cuda"), torch.tensor([f % BLOCK + n for f, (_, n) in zip(first, spans)], device="cuda"))
        many = torch.tensor([f % BLOCK + n for f, (_, n) in zip(first, spans)], device="cuda")
        back = torch.arange(len(back_who), device="cuda") - (many.cumsum(0) - many)[back_who] + torch.tensor([f - f % BLOCK for f in first], device="cuda")[back_who]
        s.update(q=_randn(g, M, heads, dim), k=_randn(g, M, kv, dim), v=_randn(g, M, kv, dim), q_out=torch.empty((M, heads, dim), device="cuda", dtype=torch.float16),
                 q_weight=_randn(g, dim, scale=0.2) + 1 if case["norm"] else None, k_weight=_randn(g, dim, scale=0.2) + 1 if case["norm"] else None,
                 rotations=_rotations(case["rot"]), positions=(torch.tensor([a for a, _ in spans], device="cuda")[who] + at).to(torch.int32), slots=slots,
                 back=table[back_who, back // page].long() * page + back % page)
        for name in ("k", "v"):
            s["pages_" + name], s[name + "_scales"] = _stored(g, pages, kv, page, dim)
            s[name + "_back"] = torch.empty((len(back), kv, dim), device="cuda", dtype=torch.float16)
        return s
    got, B = _lengths_of(case), case["B"]
    M = sum(n for _, n in got)
    width = max(1, -(-case["longest"] // page))
    table, pages = _table(g, [-(-n // page) for n, _ in got], width)
    starts = [0]
    for _, n in got:
        starts.append(starts[-1] + n)
    s.update(q=_randn(g, M, heads, dim, scale=1.5), table=table, lengths=torch.tensor([n for n, _ in got], dtype=torch.int32, device="cuda"),
             starts=None if case["kind"] == "token" else torch.tensor(starts, dtype=torch.int32, device="cuda"), rows=max(n for _, n in got),
             out=torch.empty((M, heads, dim), device="cuda", dtype=torch.float16), lse=torch.empty((M, heads), device="cuda", dtype=torch.float32))
    for name in ("k", "v"):
        if case["cache"] == "blocks":
            s["pages_" + name], s[name + "_scale"] = _stored(g, pages, kv, page, dim)
            continue
        t, by = torch.randn((pages, kv, page, dim), generator=g, device="cuda", dtype=torch.float16), None
        if case["cache"] == "heads":
            by = (torch.rand(kv, generator=g, device="cuda") + 0.5) * 0.01
            t = (t * (1.0 / by).half()[:, None, None]).clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
        s["pages_" + name], s[name + "_scale"] = t, by
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    return _blocks(s) if s["case"]["kind"] == "blocks" else _attention(s)


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


def _codes(x, e):
    """The nearest e4m3 codes of x / 2^e, as bytes."""
    return (x * torch.exp2(-e)).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_store(x, pages, scales, slots):
    """Rows x (M x kv x dim, fp32) to their slots, with the powers of their blocks brought up to date."""
    n, kv, page, dim = pages.shape
    tokens = pages.view(torch.uint8).view(n, kv, page // BLOCK, BLOCK, dim)
    block, which = torch.unique(slots // BLOCK, return_inverse=True)
    p, i = block // (page // BLOCK), block % (page // BLOCK)
    top = x.new_zeros((len(block), kv)).scatter_reduce_(0, which[:, None].expand(-1, kv), x.abs().amax(-1), "amax")
    begun = torch.zeros_like(block).scatter_reduce_(0, which, (slots % BLOCK == 0).long(), "amax") > 0
    fraction, power = torch.frexp(top)
    e = torch.where(top > 0, (power - 8 - (fraction <= TOP / 512).int()).float(), LEAST).clamp(LEAST, MOST)
    old = scales[p, :, i].float() - 127
    e = torch.where(begun[:, None], e, torch.maximum(e, old))
    was = tokens[p, :, i]
    again = _codes(was.view(torch.float8_e4m3fn).float() * torch.exp2(old)[..., None, None], e[..., None, None])
    tokens[p, :, i] = torch.where(begun[:, None, None, None], was, again)
    tokens[slots // page, :, slots % page // BLOCK, slots % BLOCK] = _codes(x, e[which][..., None])
    scales[p, :, i] = (e + 127).to(torch.uint8)


def _plain_read(pages, scales, slots):
    page = pages.shape[2]
    code = pages.view(torch.uint8)[slots // page, :, slots % page].view(torch.float8_e4m3fn).float()
    return (code * torch.exp2(scales[slots // page, :, slots % page // BLOCK].float() - 127)[..., None]).half()


def _blocks(s):
    c = s["case"]
    heads, kv, dim, page, rot = (c[k] for k in ("heads", "kv", "dim", "page", "rot"))
    if own:
        import paper_2410_21271_amd as eora
        pages = s["pages_k"].shape[0]
        eora.cache_append_blocks(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["rotations"], s["positions"], s["slots"], s["q_out"],
                                 s["pages_k"], s["pages_v"], s["k_scales"], s["v_scales"], c["M"], heads, kv, dim, heads * dim, kv * dim, kv * dim,
                                 rot, c["interleaved"], POSITIONS if rot else 0, EPS, pages, page)
        eora.cache_read(s["pages_k"], s["pages_v"], s["k_scales"], s["v_scales"], s["back"], s["k_back"], s["v_back"], len(s["back"]), kv, dim, pages, page, 8, BLOCK)
        return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
    cs = s["rotations"][s["positions"].long()] if rot else None
    q = _plain_heads(s["q"], s["q_weight"], cs, rot, c["interleaved"])
    _plain_store(_plain_heads(s["k"], s["k_weight"], cs, rot, c["interleaved"]), s["pages_k"], s["k_scales"], s["slots"])
    _plain_store(s["v"].float(), s["pages_v"], s["v_scales"], s["slots"])
    return {"q": q.half(), "k": _plain_read(s["pages_k"], s["k_scales"], s["back"]), "v": _plain_read(s["pages_v"], s["v_scales"], s["back"])}


def _attention(s):
    c = s["case"]
    B, heads, kv, dim, page, window, sinks = (c[k] for k in ("B", "heads", "kv", "dim", "page", "window", "sinks"))
    M, width, scale = s["q"].shape[0], s["table"].shape[1], dim ** -0.5
    if own:
        import paper_2410_21271_amd as eora
        if "workspace" not in s:
            s["workspace"] = eora.new_attention_rows_workspace(M, B, heads, kv, dim, width * page)
        eora.cache_attention_rows(s["q"], s["pages_k"], s["pages_v"], s["k_scale"], s["v_scale"], s["table"], s["lengths"], s["starts"], s["out"], s["lse"],
                                  M, B, heads, kv, dim, heads * dim, s["pages_k"].shape[0], page, 16 if c["cache"] == "fp16" else 8,
                                  BLOCK if c["cache"] == "blocks" else 0, width, window, sinks, scale, s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    at, rows, group = s["table"].clamp(min=0).long(), s["rows"], heads // kv

    def tokens(pages, by):
        t = pages.view(torch.uint8)[at].view(pages.dtype).float() if c["cache"] != "fp16" else pages[at].float()
        if c["cache"] == "blocks":
            t = (t.view(B, width, kv, page // BLOCK, BLOCK, dim) * torch.exp2(by[at].float() - 127)[..., None, None]).view(t.shape)
        t = t.permute(0, 2, 1, 3, 4).reshape(B, kv, width * page, dim)
        return t * by[:, None, None] if c["cache"] == "heads" else t

    # rows of each request side by side, those of shorter ones filled up with their last
    n = s["lengths"].long()
    first = torch.arange(B, device=at.device) if s["starts"] is None else s["starts"][:-1].long()
    many = torch.ones_like(n) if s["starts"] is None else (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.minimum(torch.arange(rows, device=at.device), many[:, None] - 1)
    where = first[:, None] + i
    mine, pos = (n - many)[:, None] + i, torch.arange(width * page, device=at.device)
    keep = (pos <= mine[:, :, None]) & (s["table"] >= 0).repeat_interleave(page, 1)[:, None]
    if window:
        keep &= (pos > mine[:, :, None] - window) | (pos < sinks)
    keep = keep[:, None, None]
    q = s["q"].float()[where].view(B, rows, kv, group, dim).permute(0, 2, 3, 1, 4).reshape(B, kv, group * rows, dim)
    score = torch.matmul(q, tokens(s["pages_k"], s["k_scale"]).transpose(-1, -2)).view(B, kv, group, rows, width * page).mul_(scale)
    score.masked_fill_(~keep, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, kv, group * rows, width * page), tokens(s["pages_v"], s["v_scale"])).view(B, kv, group, rows, dim) / torch.where(total == 0, 1.0, total)
    s["out"][where] = out.half().permute(0, 3, 1, 2, 4).reshape(B, rows, heads, dim)
    s["lse"][where] = (top + torch.log(total)).permute(0, 3, 1, 2, 4).reshape(B, rows, heads)
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits
def _two_to(power):
    """2^power, exactly, for whole numbers of -32 to 31."""
    return torch.tensor([2.0 ** i for i in range(-32, 32)], dtype=torch.float64, device="cuda")[power.long() + 32]


def _value(code, scales, pages, h, place):
    """The numbers that codes of tokens (page and place of each) stand for, in head h."""
    return code.double() * _two_to(scales[pages, h, place // BLOCK].long() - 127)[:, None]


def _exact_blocks(c, s):
    rot, dim, page, kv = c["rot"], c["dim"], c["page"], c["kv"]

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

    # (a key's codes have no value of their own: where 32 bits put it beside the border of two codes, either is the nearest)
    got = {"q": turned(s["q"].clone(), s["q_weight"]), "k": None}
    at = torch.full((int(s["back"].max()) + 1,), -1, dtype=torch.long, device="cuda")
    at[s["slots"]] = torch.arange(c["M"], device="cuda")
    row, block = at[s["back"]], s["back"] // BLOCK
    pages, place = s["back"] // page, s["back"] % page
    # values: those that were there, and the new ones; the least power that holds all of a block, and what it was before unless the block is begun anew
    old = torch.stack([_value(s["pages_v"].view(torch.uint8)[pages, h, place].view(torch.float8_e4m3fn), s["v_scales"], pages, h, place) for h in range(kv)], 1)
    now = torch.where((row >= 0)[:, None, None], s["v"].double()[row.clamp(min=0)], old)
    blocks, which = torch.unique(block, return_inverse=True)
    begun = torch.zeros(len(blocks), dtype=torch.bool, device="cuda")
    begun[which[(row >= 0) & (s["back"] % BLOCK == 0)]] = True
    least = torch.zeros((len(blocks), kv), dtype=torch.float64, device="cuda")
    for i in range(BLOCK):
        mine = (row >= 0) & (s["back"] % BLOCK == i)
        least[which[mine]] = torch.maximum(least[which[mine]], now[mine].abs().amax(-1))
    power = sum((least > TOP * 2.0 ** i).long() for i in range(LEAST, MOST)) + LEAST
    before = s["v_scales"][blocks * BLOCK // page, :, blocks * BLOCK % page // BLOCK].long() - 127
    by = _two_to(torch.where(begun[:, None], power, torch.maximum(power, before)))[which][..., None]
    # the nearest of the codes: three bits behind the first, down to 2^-9
    code = (now / by).clamp(-TOP, TOP)
    step = _two_to(sum((code.abs() >= 2.0 ** i).long() for i in range(-5, 9)) - 9)
    got["v"] = torch.round(code / step) * step * by
    return got


def _exact_attention(c, s):
    heads, kv, dim, page, window, sinks = (c[k] for k in ("heads", "kv", "dim", "page", "window", "sinks"))
    M, group = s["q"].shape[0], heads // kv
    out = torch.zeros((M, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((M, heads), -math.inf, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, rows) in enumerate(_lengths_of(c)):
        if n > 0:
            t = torch.arange(n, device="cuda")
            p = torch.arange(n - rows, n, device="cuda")[:, None]
            hidden = t > p
            if window:
                hidden = hidden | ((p - t >= window) & (t >= sinks))
            pages, place = s["table"][b].long()[t // page], t % page
            for h in range(kv):
                K, V = (s[x].view(torch.uint8)[pages, h, place].view(s[x].dtype) if c["cache"] != "fp16" else s[x][pages, h, place] for x in ("pages_k", "pages_v"))
                if c["cache"] == "blocks":
                    K, V = _value(K, s["k_scale"], pages, h, place), _value(V, s["v_scale"], pages, h, place)
                else:
                    K, V = (x.double() * (1.0 if by is None else by[h].double()) for x, by in ((K, s["k_scale"]), (V, s["v_scale"])))
                K = K.t().contiguous()
                for i in range(h * group, (h + 1) * group):
                    score = ((s["q"][first:first + rows, i].double() @ K) / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
                    lse[first:first + rows, i] = torch.logsumexp(score, -1)
                    out[first:first + rows, i] = torch.softmax(score, -1) @ V
        first += rows
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_blocks(case, s) if case["kind"] == "blocks" else _exact_attention(case, s)
