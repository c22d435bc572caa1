"""The attention block of examples/attention_block.py against the float64 definitions, from the rows that went in to the rows that came out.

Tolerance 12 u (u = 2^-11: fp16's unit roundoff), in oracle.linear.y_error's measure: between x and y there are ten roundings to fp16 (q, k and v from their linears, q
with its pair, q and k turned, weights, the attention's result, y, y with its pair), of 0.58 u root mean square each, and scores have a deviation of
about 1; five times their joint root mean square is 9.2 u, and y's own two are at most 2 u.
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


def exact(e, b, x, adapter):
    """y of all tokens (T x D) of a request, float64 throughout."""
    T = x.shape[0]

    def layer(l, t):
        return linear.eora_linear(t, linear.dequant(l.codes[0], l.codes[1], l.codes[2], e.GROUP), l.A, l.B)

    def own(p, t, base):
        return serving.linear_adapters(t, [(A.astype(np.float64), B.astype(np.float64)) for A, B in p.pairs], None, np.full(T, adapter), base)[0]

    x = x.astype(np.float64)
    q, k, v = own(b.pairs_q, x, layer(b.q, x)), layer(b.k, x), layer(b.v, x)
    q, k, v = serving.cache_append(q.reshape(T, e.HEADS, e.DIM), k.reshape(T, e.KV, e.DIM), v.reshape(T, e.KV, e.DIM), b.norms[0], b.norms[1], b.rotations, np.arange(T),
                                   e.DIM, False, e.EPS)
    one_page = [t.transpose(1, 0, 2)[None] for t in (k, v)]
    out = serving.cache_attention(q, one_page[0], one_page[1], np.zeros((T, 1), np.int32), np.arange(1, T + 1), 0, e.SCALE)[0].reshape(T, -1)
    return own(b.pairs_o, out, layer(b.o, out))


@pytest.mark.parametrize("prompt", [1, 21])
def test_prompt_and_tokens(example, prompt):
    import torch
    s = example.Server(8, prompt, 6)
    ys = s.prompt()
    xs, outs = [s.x_prompt], [ys]
    for i in range(6):
        xs.append(s.x.clone()[:, None])
        if i < 2:
            s.token()
            if i == 1:
                s.capture()
        else:
            s.graph.replay()
        outs.append(s.y.clone()[:, None])
    torch.cuda.synchronize()
    s.block.check()
    x, y = (torch.cat(t, 1).cpu().numpy() for t in (xs, outs))
    for i in range(s.n):
        want = exact(example, s.block, x[i], int(s.ids[i]))
        assert linear.y_error(y[i], want) <= TOLERANCE, "request %d" % i


def test_graph_gives_the_eager_bits_with_an_8_bit_cache(example):
    import torch
    results = []
    for graph in (False, True):
        s = example.Server(5, 18, 8, cache_bits=8)
        s.prompt()
        s.token()
        if graph:
            s.capture()
        ys = []
        for _ in range(7):
            s.graph.replay() if graph else s.token()
            torch.cuda.synchronize()
            ys.append(s.y.cpu().numpy())
        s.block.check()
        results.append(np.stack(ys))
    assert np.isfinite(results[0].astype(np.float64)).all()
    assert np.array_equal(results[0].view(np.uint16), results[1].view(np.uint16))
