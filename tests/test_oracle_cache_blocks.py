"""Pins of the block-scaled cache and of attention by rows in oracle/serving.py: hand-computed powers and codes, and the single-token definition."""
import numpy as np

from oracle import serving


def test_powers():
    assert serving.block_power([448.0]) == 0 and serving.block_power([448.1, 1.0]) == 1 and serving.block_power([-224.0, 0.0]) == -1
    assert serving.block_power([3.5]) == -7 and serving.block_power([np.nextafter(3.5, 4)]) == -6
    assert serving.block_power([0.0]) == -15 and serving.block_power([np.nan, np.inf, 448.0]) == 0 and serving.block_power([np.inf]) == -15
    assert serving.block_power([57344.0]) == 7 and serving.block_power([57344.1]) == 8 and serving.block_power([1e30]) == 8


def test_codes():
    # at 2^-7: 1.03125 is 132, between the codes 128 and 144; 1.0625 is 136, as far from either: the even one; 1.1875 is 152, between 144 and 160: the even one
    assert list(serving.block_codes([1.03125, 1.0625, 1.1875, 3.5, -9.0], -7)) == [128.0, 128.0, 160.0, 448.0, -448.0]
    assert list(serving.block_codes([65504.0, np.inf, 61440.0], 8)) == [240.0, 240.0, 240.0] and np.isnan(serving.block_codes([np.nan], 8))[0]
    # every code of every power is an fp16 number
    v = serving.e4m3_values()
    v = v[np.isfinite(v)]
    for e in range(-15, 9):
        x = v[np.abs(v) <= (240 if e == 8 else 448)] * 2.0 ** e
        assert np.array_equal(x, x.astype(np.float16).astype(np.float64))


def test_append_grows_and_begins_anew():
    codes, powers = np.zeros((2, 1, 16, 4)), np.full((2, 1, 1), -15)
    row = lambda x: np.full((1, 1, 4), float(x))          # noqa: E731
    serving.cache_append_blocks(row(3.5), [16], codes, powers)
    assert powers[1, 0, 0] == -7 and codes[1, 0, 0, 0] == 448 and powers[0, 0, 0] == -15
    serving.cache_append_blocks(row(1.0), [17], codes, powers)
    assert powers[1, 0, 0] == -7 and codes[1, 0, 1, 0] == 128
    serving.cache_append_blocks(row(28.0), [18], codes, powers)            # eight times as much: codes an eighth
    assert powers[1, 0, 0] == -4 and list(codes[1, 0, :4, 0]) == [56, 16, 448, 0]
    serving.cache_append_blocks(row(0.5), [16], codes, powers)             # token 0: anew
    assert powers[1, 0, 0] == -9 and codes[1, 0, 0, 0] == 256
    serving.cache_append_blocks(np.concatenate([row(2), row(9)]), [-1, 32], codes, powers)
    assert powers[0, 0, 0] == -15 and not codes[0].any()


def test_rows_are_single_tokens_of_their_lengths():
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(4, 2, 16, 8)), rng.normal(size=(4, 2, 16, 8))
    table = np.array([[2, 0], [1, 3], [3, -1]])
    q = rng.normal(size=(9, 4, 8))
    out, lse, size, most, logit = serving.cache_attention_rows(q, k, v, table, [20, 3, 18], [0, 5, 5, 8], 0, 0, 0.3)
    assert np.isnan(out[8]).all() and np.isnan(lse[8]).all()
    for b, rows, n in ((0, range(5), 20), (2, range(5, 8), 18)):
        for i, m in enumerate(rows):
            ref = serving.cache_attention(q[m:m + 1], k, v, table[b:b + 1], [n - len(rows) + i + 1], 0, 0.3)
            for got, want in zip((out, lse, size, most, logit), ref):
                assert np.allclose(got[m], want[0])
    # a window: without first tokens as there; with them, the whole where they meet
    for window in (1, 4, 30):
        one = serving.cache_attention_rows(q[:3], k, v, table, [20, 3, 18], None, window, 0, 0.3)
        ref = serving.cache_attention(q[:3], k, v, table, [20, 3, 18], window, 0.3)
        assert all(np.allclose(x, y) for x, y in zip(one, ref))
    assert np.allclose(serving.cache_attention_rows(q[:1], k, v, table[:1], [20], None, 4, 16, 0.3)[0], serving.cache_attention(q[:1], k, v, table[:1], [20], 0, 0.3)[0])
    # first tokens: the softmax over those, by hand
    got = serving.cache_attention_rows(q[:1], k, v, table[:1], [20], [0, 1], 2, 3, 0.3)
    K, V = (np.concatenate([t[2, 1, :3], t[0, 1, 2:4]]) for t in (k, v))
    s = np.exp(0.3 * (K @ q[0, 3]))
    assert np.allclose(got[0][0, 3], s @ V / s.sum()) and np.allclose(got[1][0, 3], np.log(s.sum()))
    # more rows than tokens: the first see nothing
    out, lse = serving.cache_attention_rows(q[:4], k, v, table[:1], [2], [0, 4], 0, 0, 0.3)[:2]
    assert not out[:2].any() and np.all(lse[:2] == -np.inf) and np.allclose(out[2, 0], v[2, 0, 0])
