"""Pins of oracle/serving.py: hand-computed 8-bit values, torch's own 8-bit type, closed forms."""
import math

import numpy as np
import torch

from oracle import serving


def test_e4m3_values_and_nearest():
    v = serving.e4m3_values()
    assert v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7E] == 448.0 and v[0xB8] == -1.0 and math.isnan(v[0x7F])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True)
    x = np.concatenate([np.random.default_rng(1).normal(0, s, 4000) for s in (1e-3, 0.1, 20.0)] + [(v[:126] + v[1:127]) / 2, v[:127], [0.0, -0.0, 448.0]])
    x32 = x.astype(np.float32)
    ref = torch.from_numpy(x32).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(serving.e4m3_nearest(x32), ref)
    assert list(serving.e4m3_nearest([500.0, -1e9, np.inf])) == [448.0, -448.0, 448.0] and np.isnan(serving.e4m3_nearest([np.nan]))[0]


def test_adapters_brute_force():
    rng = np.random.default_rng(2)
    pairs = [(rng.integers(-3, 4, (2, 5)).astype(float), rng.integers(-3, 4, (4, 2)).astype(float)) for _ in range(3)]
    x, base = rng.integers(-3, 4, (6, 5)).astype(float), rng.integers(-3, 4, (6, 4)).astype(float)
    ids, s = [0, 2, -1, 3, 1, 2], [1.0, 0.5, 2.0]
    y, size = serving.linear_adapters(x, pairs, s, ids, base)
    for m, a in enumerate(ids):
        for o in range(4):
            want = base[m, o]
            if 0 <= a < 3:
                want += s[a] * sum(pairs[a][1][o, c] * sum(pairs[a][0][c, i] * x[m, i] for i in range(5)) for c in range(2))
            assert y[m, o] == want and size[m, o] >= abs(want)


def test_head_norm_and_rotation():
    x = np.array([3.0, 4.0, 0.0, 0.0])
    assert np.allclose(serving.head(x, np.array([1.0, 2.0, 1.0, 1.0]), 0.0, None, 0, False), [3 / 2.5, 8 / 2.5, 0, 0])
    quarter = [(0.0, 1.0), (1.0, 0.0)]                    # the first pair by 90 degrees, the second not at all
    assert np.array_equal(serving.head(x, None, 0.0, quarter, 4, False), [0.0, 4.0, 3.0, 0.0])
    assert np.array_equal(serving.head(x, None, 0.0, quarter, 4, True), [-4.0, 3.0, 0.0, 0.0])
    # a rotation keeps the scalar product of two heads turned by angles of the same difference
    rng = np.random.default_rng(3)
    a, b, f = rng.normal(size=8), rng.normal(size=8), rng.normal(size=4)
    turn = lambda p: np.stack((np.cos(p * f), np.sin(p * f)), -1)       # noqa: E731
    for inter in (False, True):
        dots = [serving.head(a, None, 0.0, turn(p + 3), 8, inter) @ serving.head(b, None, 0.0, turn(p), 8, inter) for p in (0, 5, 11)]
        assert np.allclose(dots, dots[0])


def test_attention_closed_forms():
    rng = np.random.default_rng(4)
    k, v = rng.normal(size=(3, 2, 4, 8)), rng.normal(size=(3, 2, 4, 8))
    table = np.array([[2, 0], [1, -1], [0, 1]])
    zero = np.zeros((3, 4, 8))
    out, lse, size, _, _ = serving.cache_attention(zero, k, v, table, [6, 3, 0], 0, 0.5)      # no scores: means
    rows = np.concatenate([v[2, 1], v[0, 1, :2]])
    assert np.allclose(out[0, 2], rows.mean(0)) and np.allclose(lse[0], math.log(6)) and np.allclose(out[1, 0], v[1, 0, :3].mean(0))
    assert not out[2].any() and np.all(lse[2] == -np.inf) and np.all(size >= np.abs(out) - 1e-12)
    q = rng.normal(size=(1, 4, 8))
    out, lse, _, _, _ = serving.cache_attention(q, k, v, table[:1], [8], 1, 0.5)              # one token in the window: its value
    assert np.allclose(out[0, 3], v[0, 1, 3]) and np.allclose(lse[0, 3], 0.5 * q[0, 3] @ k[0, 1, 3])
    # a torch softmax over all of them
    out, lse, _, _, _ = serving.cache_attention(q, k, v, table[:1], [7], 0, 0.3)
    K, V = (np.concatenate([t[2, 1], t[0, 1, :3]]) for t in (k, v))
    s = torch.from_numpy(0.3 * (q[0, 2:] @ K.T))
    assert np.allclose(out[0, 2:], torch.softmax(s, -1).numpy() @ V) and np.allclose(lse[0, 2:], torch.logsumexp(s, -1).numpy())
    # a missing page masks its tokens only
    out, _, _, _, _ = serving.cache_attention(q, k, v, np.array([[5, 0]]), [7], 0, 0.3)
    ref, _, _, _, _ = serving.cache_attention(q, k, v, np.array([[0]]), [3], 0, 0.3)
    assert np.allclose(out, ref)
