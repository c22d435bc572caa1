"""examples/attention_block.py with scales for blocks of the cache, a window and first tokens that stay visible, against the float64 definitions.

What the cache holds is read back after each step, and the definitions take keys and values from there: so its 8 bits are no part of the error.  Tolerance as
in the test of the example's other options, 12 u (u = 2^-11) in oracle.linear.y_error's measure: between x and y there are at most ten roundings to fp16.
"""
import importlib.util
import os

import numpy as np
import pytest

from oracle import linear, serving

pytestmark = pytest.mark.gpu
TOLERANCE = 12 * 2.0 ** -11


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def exact(e, b, x, adapter, first, k, v):
    """y of tokens first, first + 1, ... of a request (T x D), float64, over the keys and values that it has (tokens x KV x DIM)."""
    T, n = x.shape[0], len(k)
    assert n == first + T

    def layer(l, t):
        return linear.eora_linear(t, linear.dequant(l.codes[0], l.codes[1], l.codes[2], e.GROUP), l.A, l.B)

    def own(p, t, base):
        return serving.linear_adapters(t, [(A.astype(np.float64), B.astype(np.float64)) for A, B in p.pairs], None, np.full(T, adapter), base)[0]

    x = x.astype(np.float64)
    q = own(b.pairs_q, x, layer(b.q, x)).reshape(T, e.HEADS, e.DIM)
    nothing = np.zeros((T, e.KV, e.DIM))
    q = serving.cache_append(q, nothing, nothing, b.norms[0], b.norms[1], b.rotations, np.arange(first, n), e.DIM, False, e.EPS)[0]
    width = -(-n // 16)
    pages = [np.zeros((width, e.KV, 16, e.DIM)) for _ in range(2)]
    for t in range(n):
        pages[0][t // 16, :, t % 16], pages[1][t // 16, :, t % 16] = k[t], v[t]
    out = serving.cache_attention_rows(q, pages[0], pages[1], np.arange(width)[None], [n], [0, T], b.window, b.sinks, e.SCALE)[0].reshape(T, -1)
    return own(b.pairs_o, out, layer(b.o, out))


@pytest.mark.parametrize("bits, options", [(16, dict(window=17, sinks=3)), (8, dict(block_scales=True)), (8, dict(block_scales=True, window=20, sinks=5)), (8, dict(window=9))])
def test_prompts_and_tokens(example, bits, options):
    import torch
    s = example.Server(5, 37, 12, bits, **options)
    b = s.block

    def compare(x, y, first):
        torch.cuda.synchronize()
        b.check()
        for i in range(s.n):
            k, v = (t.cpu().numpy().astype(np.float64) for t in b.cached(i, first + x.shape[1]))
            want = exact(example, b, x[i].cpu().numpy(), int(s.ids[i]), first, k, v)
            assert linear.y_error(y[i].cpu().numpy(), want) <= TOLERANCE, "request %d, tokens from %d" % (i, first)

    compare(s.x_prompt, s.prompt(), 0)
    for i in range(12):                                  # from the third on by replays; the block of token 48 is begun in the last
        x = s.x.clone()
        if i < 2:
            s.token()
        else:
            if i == 2:
                s.capture()
            s.graph.replay()
        if i in (0, 1, 2, 5, 11):
            compare(x[:, None], s.y[:, None], 37 + i)
        else:
            torch.cuda.synchronize()
