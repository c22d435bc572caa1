"""The attention half of a decoder layer, served to requests that have adapters of their own and share a paged cache.

    python examples/attention_block.py [--requests 8] [--prompt 40] [--tokens 64] [--cache-bits 8]

Six calls a step:  q, k, v = compensated 4-bit linears of x (one launch)  ->  q += the request's own pair  ->  norm, rotation and store into the
cache  ->  attention over the request's pages  ->  compensated output linear, += the request's own pair.  A prompt is a step whose rows are its
tokens, each with the length that it may see; tokens after it are generated by replays of one captured graph, which
moves positions, slots and lengths on by itself.  Weights and inputs are drawn.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_21271_amd as eora  # noqa: E402
import synth  # noqa: E402

D, HEADS, KV, DIM, PAGE = 1024, 16, 4, 64, 16
RANK, W_BITS, GROUP = 64, 4, 128                     # of the layer: compensation and backbone
PAIR_RANK, PAIRS = 32, 6                             # of the requests' own pairs
EPS, SCALE = 1e-6, DIM ** -0.5


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Linear:
    """A compensated compressed linear layer as stored."""

    def __init__(self, seed, d_in, d_out):
        W, A, B, _ = synth.draw_layer(seed, d_in, d_out, 1, RANK)
        self.codes = synth.quantize_rtn(W, W_BITS, GROUP)
        self.A, self.B, self.d_in, self.d_out = A, B, d_in, d_out
        qweight, qzeros, scales = eora.pack_q(self.codes[0], self.codes[1], self.codes[2], W_BITS, GROUP)
        self.stored = [dev(t) for t in (qweight, scales, qzeros, eora.pack_factor_f16(A), eora.pack_factor_f16(B))]

    def member(self, y):
        return tuple(self.stored) + (None, None, y, self.d_out)


class Pairs:
    """The requests' low-rank pairs beside one linear: a slot each in two pools."""

    def __init__(self, seed, d_in, d_out):
        rng = np.random.default_rng(seed)
        self.pairs = [((0.02 * rng.standard_normal((PAIR_RANK, d_in))).astype(np.float16), (0.1 * rng.standard_normal((d_out, PAIR_RANK))).astype(np.float16))
                      for _ in range(PAIRS)]
        self.A = dev(np.concatenate([eora.pack_factor_f16(a) for a, _ in self.pairs]))
        self.B = dev(np.concatenate([eora.pack_factor_f16(b) for _, b in self.pairs]))


class Block:
    def __init__(self, requests, most_tokens, most_rows, cache_bits=16, seed=7):
        self.q, self.k, self.v, self.o = (Linear(seed + i, D, n) for i, n in enumerate((HEADS * DIM, KV * DIM, KV * DIM, D)))
        self.pairs_q, self.pairs_o = Pairs(seed + 4, D, HEADS * DIM), Pairs(seed + 5, HEADS * DIM, D)
        rng = np.random.default_rng(seed + 6)
        self.norms = [(1 + 0.1 * rng.standard_normal(DIM)).astype(np.float16) for _ in range(2)]
        self.d_norms = [dev(t) for t in self.norms]
        angle = np.arange(most_tokens)[:, None] * 10000.0 ** (-np.arange(DIM // 2) / (DIM // 2))
        self.rotations = np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)
        self.d_rotations = dev(self.rotations)
        # the cache: pages handed out in an order of their own
        self.bits, self.width = cache_bits, (most_tokens + PAGE - 1) // PAGE
        self.n_pages, self.most_tokens = requests * self.width, most_tokens
        kind = torch.float16 if cache_bits == 16 else torch.uint8
        self.pages = [torch.zeros((self.n_pages, KV, PAGE, DIM), dtype=kind, device="cuda") for _ in range(2)]
        # what a code of 1 stands for: keys are normed, so a few units at most; values have a deviation of 0.7
        self.scales = [torch.full((KV,), s, device="cuda") for s in (0.02, 0.01)] if cache_bits == 8 else [None, None]
        self.table = dev(rng.permutation(self.n_pages).astype(np.int32).reshape(requests, self.width))
        self.w_layer = eora.new_workspace(most_rows, D, D, RANK, n_members=3)
        self.w_pairs = eora.new_adapters_workspace(most_rows, D, D, PAIR_RANK)
        self.w_attention = eora.new_attention_workspace(most_rows, HEADS, KV, DIM, self.width * PAGE)

    def slots(self, request, positions):
        return self.table[request.long(), (positions // PAGE).long()].long() * PAGE + positions % PAGE

    def __call__(self, x, y, ids, positions, slots, lengths, table):
        """x, y: rows x D; row m is token positions[m] of a request with the pages table[m], and sees lengths[m] tokens."""
        M = x.shape[0]
        q, k, v = (torch.empty((M, n * DIM), dtype=torch.float16, device="cuda") for n in (HEADS, KV, KV))
        eora.linear_q_group(x, [self.q.member(q), self.k.member(k), self.v.member(v)], M, D, RANK, W_BITS, GROUP, 16, self.w_layer)
        eora.linear_adapters(x, self.pairs_q.A, self.pairs_q.B, None, None, None, None, ids, q, q, M, D, HEADS * DIM, PAIR_RANK, PAIRS, 16, self.w_pairs)
        eora.cache_append(q, k, v, self.d_norms[0], self.d_norms[1], self.d_rotations, positions, slots, q, self.pages[0], self.pages[1], self.scales[0],
                          self.scales[1], M, HEADS, KV, DIM, HEADS * DIM, KV * DIM, KV * DIM, DIM, False, self.most_tokens, EPS, self.n_pages, PAGE, self.bits)
        out = torch.empty_like(q)
        eora.cache_attention(q, self.pages[0], self.pages[1], self.scales[0], self.scales[1], table, lengths, out, None, M, HEADS, KV, DIM, HEADS * DIM,
                             self.n_pages, PAGE, self.bits, self.width, 0, SCALE, self.w_attention)
        o = self.o
        eora.linear_q(out, *o.stored, None, None, y, M, o.d_in, o.d_out, RANK, W_BITS, GROUP, 16, self.w_layer)
        eora.linear_adapters(out, self.pairs_o.A, self.pairs_o.B, None, None, None, None, ids, y, y, M, o.d_in, o.d_out, PAIR_RANK, PAIRS, 16, self.w_pairs)

    def check(self):
        eora.workspace_error(self.w_layer)
        eora.workspace_error(self.w_pairs)


def following(x, y):
    """The next token's input from this one's output (stands for the rest of the layer): a normed residual."""
    z = x.float() + y.float()
    return (z * torch.rsqrt(z.square().mean(-1, keepdim=True) + EPS)).half()


class Server:
    """Requests with one prompt length, each with an adapter or none."""

    def __init__(self, requests, prompt, tokens, cache_bits=16):
        self.n, self.prompt_tokens = requests, prompt
        self.block = Block(requests, prompt + tokens, max(requests, prompt), cache_bits)
        rng = np.random.default_rng(3)
        self.x_prompt = dev(rng.standard_normal((requests, prompt, D)).astype(np.float16))
        self.ids = torch.arange(requests, dtype=torch.int32, device="cuda") % (PAIRS + 1) - 1       # -1: no adapter
        self.request = torch.arange(requests, dtype=torch.int32, device="cuda")
        self.x = torch.empty((requests, D), dtype=torch.float16, device="cuda")
        self.y = torch.empty_like(self.x)
        self.positions = torch.full((requests,), prompt, dtype=torch.int32, device="cuda")
        self.graph = None

    def prompt(self):
        """All prompts, one after the other; returns y of their tokens."""
        P, b = self.prompt_tokens, self.block
        places = torch.arange(P, dtype=torch.int32, device="cuda")
        ys = torch.empty_like(self.x_prompt)
        for i in range(self.n):
            request = self.request[i].expand(P).contiguous()
            b(self.x_prompt[i], ys[i], self.ids[i].expand(P).contiguous(), places, b.slots(request, places), places + 1, b.table[i].expand(P, -1).contiguous())
        self.x.copy_(following(self.x_prompt[:, -1], ys[:, -1]))
        return ys

    def token(self):
        b = self.block
        b(self.x, self.y, self.ids, self.positions, b.slots(self.request, self.positions), self.positions + 1, b.table)
        self.x.copy_(following(self.x, self.y))
        self.positions.add_(1)

    def capture(self):
        """One token as a graph (the first is run as it is, outside)."""
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.token()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--cache-bits", type=int, default=16, choices=(16, 8))
    args = ap.parse_args()
    s = Server(args.requests, args.prompt, args.tokens, args.cache_bits)
    s.prompt()
    s.token()
    s.capture()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(args.tokens - 1):
        s.graph.replay()
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    s.block.check()
    assert torch.isfinite(s.y).all()
    if args.tokens > 1:
        print("%d requests, prompts of %d tokens, %d bits a cached value: %.1f us a token of each" % (args.requests, args.prompt, args.cache_bits, took * 1e6 / (args.tokens - 1)))


if __name__ == "__main__":
    main()
