"""What eora_cache_append_blocks, eora_cache_read and eora_cache_attention_rows refuse, and with which code, before anything is enqueued:
the calls need no GPU, their pointers are never followed."""
import pytest

import paper_2410_21271_amd as eora
from tests.test_serving_refusals import ALIGN, BIG, G, INF, NAN, NULL, OK, SHAPE, UNSUPPORTED, VALUE, WORKSPACE, call

APPEND = dict(q=G, k=G, v=G, qw=None, kw=None, rot_table=G, positions=G, slots=G, q_out=G, pk=G, pv=G, ks=G + 1, vs=G + 3, M=4, heads=8, kv=2, dim=64,
              q_stride=512, k_stride=128, v_stride=128, rot=64, interleaved=0, n_positions=100, eps=1e-5, n_pages=4, page=16, stream=None)
READ = dict(pk=G, pv=G, ks=None, vs=None, slots=G, k=G, v=G, M=4, kv=2, dim=64, n_pages=4, page=16, bits=16, block=0, stream=None)
ROWS = dict(q=G, pk=G, pv=G, ks=None, vs=None, table=G, lengths=G, starts=G, out=G, lse=None, M=30, B=3, heads=8, kv=2, dim=64, q_stride=512, n_pages=4, page=16,
            bits=16, block=0, width=8, window=0, sinks=0, scale=0.125, ws=G, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(slots=None)), (NULL, dict(q_out=None)), (NULL, dict(pk=None)), (NULL, dict(pv=None)),
    (NULL, dict(ks=None)), (NULL, dict(vs=None)), (NULL, dict(rot_table=None)), (NULL, dict(positions=None)),
    (UNSUPPORTED, dict(dim=96, q_stride=768, k_stride=192, v_stride=192)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(kv=0)), (SHAPE, dict(q_stride=504)), (SHAPE, dict(q_stride=516)), (SHAPE, dict(k_stride=120)),
    (SHAPE, dict(v_stride=132)), (SHAPE, dict(rot=8)), (SHAPE, dict(rot=80)), (SHAPE, dict(n_positions=0)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(page=24)),
    (SHAPE, dict(n_pages=2 ** 27, page=16)), (VALUE, dict(qw=G, eps=-1.0)), (VALUE, dict(kw=G, eps=NAN)),
    (ALIGN, dict(q=G + 8)), (ALIGN, dict(kw=G + 2)), (ALIGN, dict(q_out=G + 8)), (ALIGN, dict(pk=G + 8)), (ALIGN, dict(positions=G + 2)), (ALIGN, dict(slots=G + 4)),
    (OK, dict(M=0)), (OK, dict(M=0, rot=0, rot_table=None, positions=None, n_positions=0)),
])
def test_append_blocks(code, kw):
    assert call(eora.lib.eora_cache_append_blocks, APPEND, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(pk=None)), (NULL, dict(pv=None)), (NULL, dict(slots=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(bits=8)),
    (NULL, dict(bits=8, block=16, ks=G)), (UNSUPPORTED, dict(bits=4)), (UNSUPPORTED, dict(block=16)), (UNSUPPORTED, dict(bits=8, block=32, ks=G, vs=G)),
    (UNSUPPORTED, dict(bits=8, block=-16, ks=G, vs=G)), (UNSUPPORTED, dict(dim=32)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(kv=0)), (SHAPE, dict(page=8)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(kv=2 ** 26)),
    (ALIGN, dict(k=G + 8)), (ALIGN, dict(v=G + 2)), (ALIGN, dict(slots=G + 4)), (ALIGN, dict(bits=8, ks=G + 1, vs=G)),
    (OK, dict(M=0)), (OK, dict(M=0, bits=8, block=16, ks=G + 1, vs=G + 1)),
])
def test_read(code, kw):
    assert call(eora.lib.eora_cache_read, READ, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(q=None)), (NULL, dict(table=None)), (NULL, dict(lengths=None)), (NULL, dict(out=None)), (NULL, dict(pk=None)), (NULL, dict(pv=None)),
    (NULL, dict(bits=8, vs=G)), (UNSUPPORTED, dict(bits=32)), (UNSUPPORTED, dict(block=16)), (UNSUPPORTED, dict(bits=8, block=8, ks=G, vs=G)),
    (UNSUPPORTED, dict(dim=32, q_stride=256)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(B=-1)), (SHAPE, dict(B=8193)), (SHAPE, dict(starts=None)), (SHAPE, dict(heads=7, q_stride=448)), (SHAPE, dict(heads=0)), (SHAPE, dict(kv=0)),
    (SHAPE, dict(width=0)), (SHAPE, dict(window=-1)), (SHAPE, dict(sinks=-1)), (SHAPE, dict(q_stride=511)), (SHAPE, dict(page=8)), (SHAPE, dict(width=2 ** 26 + 1)),
    (SHAPE, dict(M=2 ** 30)), (SHAPE, dict(n_pages=2 ** 26, heads=64, kv=64, q_stride=64 * 64)), (SHAPE, dict(M=8192, starts=None, B=8192, heads=2 ** 12, kv=2 ** 12, q_stride=2 ** 18, width=128)),
    (VALUE, dict(scale=NAN)), (VALUE, dict(scale=-INF)),
    (ALIGN, dict(q=G + 2)), (ALIGN, dict(out=G + 8)), (ALIGN, dict(table=G + 2)), (ALIGN, dict(lengths=G + 1)), (ALIGN, dict(starts=G + 2)), (ALIGN, dict(lse=G + 2)),
    (ALIGN, dict(ws=G + 4)), (ALIGN, dict(bits=8, ks=G + 2, vs=G)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=eora.cache_attention_rows_workspace_bytes(30, 3, 8, 2, 64, 128) - 1)),
    (OK, dict(B=0)), (OK, dict(M=0)), (OK, dict(M=0, B=0, starts=None)), (OK, dict(M=0, bits=8, block=16, ks=G + 1, vs=G + 1)),
])
def test_attention_rows(code, kw):
    assert call(eora.lib.eora_cache_attention_rows, ROWS, **kw) == code


def test_workspace_sizes():
    t = eora.cache_attention_rows_workspace_bytes
    assert t(-1, 3, 8, 2, 64, 128) == 0 and t(3, 8193, 8, 2, 64, 128) == 0 and t(3, 3, 7, 2, 64, 128) == 0 and t(3, 3, 8, 2, 96, 128) == 0
    for heads, kv, dim in ((8, 8, 64), (8, 1, 128), (40, 2, 256)):
        sizes = [t(0, 0, heads, kv, dim, 0), t(1, 1, heads, kv, dim, 16), t(64, 5, heads, kv, dim, 4096), t(10 ** 6, 8192, heads, kv, dim, 1 << 17)]
        assert 0 < sizes[0] and sizes == sorted(sizes)
        assert eora.cache_attention_workspace_bytes(8192, heads, kv, dim, 1 << 17) <= sizes[-1]
    assert t(1, 1, 8, 2, 64, 16) <= t(1, 1, 8, 2, 128, 16) <= t(1, 1, 8, 2, 256, 16)


@pytest.mark.gpu                                         # (the binding asks torch for its stream)
def test_binding_raises_with_the_code():
    with pytest.raises(eora.EoraError) as e:
        eora.cache_append_blocks(*[None] * 13, 1, 8, 2, 64, 512, 128, 128, 64, False, 100, 0.0, 4, 16)
    assert e.value.status == NULL and "cache_append_blocks" in str(e.value)
    with pytest.raises(eora.EoraError) as e:
        eora.cache_read(*[None] * 7, 1, 2, 64, 4, 16, 16, 0)
    assert e.value.status == NULL
    with pytest.raises(eora.EoraError) as e:
        eora.cache_attention_rows(*[None] * 10, 30, 3, 8, 2, 64, 512, 4, 16, 16, 0, 8, 0, 0, 0.125, None)
    assert e.value.status == NULL
