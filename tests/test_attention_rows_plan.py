"""How eora_cache_attention_rows deals out tiles of rows and of keys to workgroups, found on the host (no GPU): all of the work once, in bounds whatever row_starts say."""
import numpy as np
import pytest

import paper_2410_21271_amd as eora
from tests.test_serving_refusals import NULL, OK, SHAPE, UNSUPPORTED

ROOM = 576                                    # partial results that a workspace has room for


def unit(requests, heads, kv, dim, page, bits, width, window, sinks, i, starts=None, M=None):
    lengths = np.array([n for n, _ in requests], np.int32)
    starts = np.cumsum([0] + [r for _, r in requests]).astype(np.int32) if starts is None else starts
    return eora.debug_attention_rows_unit(lengths, starts, int(starts[-1]) if M is None else M, heads, kv, dim, page, bits, width, window, sinks, i)


CASES = [
    # tokens and rows of the requests, heads, kv, dim, bits, window, sinks
    ([(17, 17)], 32, 8, 128, 16, 0, 0),
    ([(2048, 2048)], 32, 8, 128, 8, 0, 0),
    ([(3000, 3), (20, 20), (0, 2), (5, 0)], 4, 2, 64, 16, 0, 0),
    ([(2000, 2)] + [(7, 7)] * 75, 256, 1, 64, 16, 900, 5),
    ([(3001, 500), (1200, 37), (900, 1)] * 3, 15, 3, 64, 16, 1000, 37),
    ([(4000, 300), (100, 100)], 16, 2, 256, 16, 0, 0),
    ([(60, 40)] * 40 + [(900, 90)] + [(5, 0), (0, 0)] * 10 + [(1500, 1)] * 9, 8, 2, 128, 8, 0, 0),
    ([(9000, 3)] + [(20, 2)] * 90, 4, 1, 64, 16, 300, 4),
    ([(i % 5, i % 3) for i in range(200)], 2, 1, 64, 16, 0, 0),
]


@pytest.mark.parametrize("requests,heads,kv,dim,bits,window,sinks", CASES)
def test_all_of_the_work_once(requests, heads, kv, dim, bits, window, sinks):
    group, width = heads // kv, -(-max(n for n, _ in requests) // 16)
    args = (requests, heads, kv, dim, 16, bits, width, window, sinks)
    narrow, workgroups = unit(*args, 0)[:2]
    TQ, KT = (32, 32) if narrow else (128, 64)
    steps, parts_of, places, seen_parts = {}, {}, set(), set()
    for i in range(workgroups):
        _, _, b, h, tile, tiles, part, parts, n, place = unit(*args, i)
        if b < 0:
            continue
        assert tiles == -(-requests[b][1] * group // TQ) and 0 <= tile < tiles and 0 <= h < kv and 0 <= part < parts
        assert (b, h, tile, part) not in seen_parts
        seen_parts.add((b, h, tile, part))
        assert parts_of.setdefault((b, h, tile), parts) == parts
        steps[b, h, tile] = steps.get((b, h, tile), 0) + n
        assert (place >= 0) == (parts > 1) and place < ROOM
        if place >= 0:
            assert place not in places
            places.add(place)
    for key, parts in parts_of.items():
        assert all(key + (p,) in seen_parts for p in range(parts))
    for b, (n, rows) in enumerate(requests):
        for tile in range(-(-rows * group // TQ)):
            low, high = n - rows + tile * TQ // group, n - rows + (min((tile + 1) * TQ, rows * group) - 1) // group
            t = np.arange(max(0, high + 1))
            t = t[(t > low - window) | (t < sinks)] if window else t
            for h in range(kv):
                assert steps[b, h, tile] == len(np.unique(t // KT))


@pytest.mark.parametrize("B", [64, 65, 8192])
def test_rows_that_decrease(B):
    """Requests that share all rows, many times 2^32 units of work in all: what a workgroup finds is a tile that there is."""
    M, heads = 1 << 20, 128
    for first in (0, B // 2 - 1):                         # requests without a row before
        starts = np.zeros(B + 1, np.int32)
        starts[first + 1::2] = M
        requests = [(4096, 0)] * B
        args = (requests, heads, 1, 64, 16, 16, 256, 0, 0)
        _, workgroups = unit(*args, 0, starts, M)[:2]
        for i in list(range(0, workgroups, workgroups // 50)) + [workgroups - 1]:
            _, _, b, h, tile, tiles, part, parts, n, place = unit(*args, i, starts, M)
            assert 0 <= b < B and starts[b + 1] > starts[b] and tiles == M and 0 <= tile < tiles and h == 0 and 0 <= part < parts and place < ROOM


def test_refusals():
    n, s = np.array([10], np.int32), np.array([0, 5], np.int32)
    good = (5, 4, 2, 64, 16, 16, 1, 0, 0, 0)
    assert len(eora.debug_attention_rows_unit(n, s, *good)) == 10
    for status, at, value in ((SHAPE, 0, 0), (SHAPE, 1, 3), (UNSUPPORTED, 3, 96), (SHAPE, 4, 8), (UNSUPPORTED, 5, 4), (SHAPE, 6, 0), (SHAPE, 7, -1), (SHAPE, 8, -1), (SHAPE, 9, -1), (SHAPE, 0, 1 << 30)):
        with pytest.raises(eora.EoraError) as e:
            eora.debug_attention_rows_unit(n, s, *good[:at], value, *good[at + 1:])
        assert e.value.status == status
    assert eora.lib.eora_debug_attention_rows_unit(None, None, 5, 1, *good[1:], None) == NULL and OK == 0
