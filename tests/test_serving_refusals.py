"""What eora_linear_adapters, eora_cache_append and eora_cache_attention refuse, and with which code, before anything is enqueued:
the calls need no GPU, their pointers are never followed."""
import pytest

import paper_2410_21271_amd as eora

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, VALUE = 0, -1, -2, -3, -4, -5, -7
G = 0x1000                                               # an aligned address
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")

ADAPTERS = dict(x=G, A=G, B=G, As=None, Bs=None, ranks=None, scalings=None, ids=G, base=None, y=G, M=4, d_in=256, d_out=32, r=64, n=3, bits=16,
                ws=G, ws_bytes=BIG, stream=None)
APPEND = dict(q=G, k=G, v=G, qw=None, kw=None, rot_table=G, positions=G, slots=G, q_out=G, pk=G, pv=G, ks=None, vs=None, M=4, heads=8, kv=2, dim=64,
              q_stride=512, k_stride=128, v_stride=128, rot=64, interleaved=0, n_positions=100, eps=1e-5, n_pages=4, page=16, bits=16, stream=None)
ATTENTION = dict(q=G, pk=G, pv=G, ks=None, vs=None, table=G, lengths=G, out=G, lse=None, B=3, heads=8, kv=2, dim=64, q_stride=512, n_pages=4, page=16,
                 bits=16, width=8, window=0, scale=0.125, ws=G, ws_bytes=BIG, stream=None)


def call(fn, defaults, **kw):
    assert not set(kw) - set(defaults)
    return fn(*{**defaults, **kw}.values())


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(x=None)), (NULL, dict(A=None)), (NULL, dict(B=None)), (NULL, dict(ids=None)), (NULL, dict(y=None)),
    (NULL, dict(bits=4, r=128, As=G)), (NULL, dict(bits=3, r=128, Bs=G)),
    (UNSUPPORTED, dict(bits=8)), (UNSUPPORTED, dict(bits=0)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(d_in=0)), (SHAPE, dict(d_in=192)), (SHAPE, dict(d_out=40)), (SHAPE, dict(d_out=0)), (SHAPE, dict(n=0)),
    (SHAPE, dict(r=0)), (SHAPE, dict(r=48)), (SHAPE, dict(r=544)), (SHAPE, dict(bits=4, r=96, As=G, Bs=G)), (SHAPE, dict(bits=3, r=64, As=G, Bs=G)),
    (ALIGN, dict(x=G + 8)), (ALIGN, dict(base=G + 2)), (ALIGN, dict(y=G + 4)), (ALIGN, dict(ids=G + 2)), (ALIGN, dict(ranks=G + 1)), (ALIGN, dict(ws=G + 8)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=eora.adapters_workspace_bytes(4, 256, 32, 64) - 1)),
    (OK, dict(M=0)), (OK, dict(M=0, bits=4, r=64, As=G, Bs=G)),
])
def test_adapters(code, kw):
    assert call(eora.lib.eora_linear_adapters, ADAPTERS, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(slots=None)), (NULL, dict(q_out=None)), (NULL, dict(pk=None)), (NULL, dict(pv=None)),
    (NULL, dict(rot_table=None)), (NULL, dict(positions=None)), (NULL, dict(bits=8, ks=G)), (NULL, dict(bits=8, vs=G)),
    (UNSUPPORTED, dict(bits=4)), (UNSUPPORTED, dict(dim=96, q_stride=768, k_stride=192, v_stride=192)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(heads=0)), (SHAPE, dict(kv=0)), (SHAPE, dict(q_stride=504)), (SHAPE, dict(q_stride=516)), (SHAPE, dict(k_stride=120)),
    (SHAPE, dict(v_stride=132)), (SHAPE, dict(heads=2 ** 26, q_stride=2 ** 31 - 8)), (SHAPE, dict(rot=8)), (SHAPE, dict(rot=80)), (SHAPE, dict(rot=-16)),
    (SHAPE, dict(n_positions=0)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(page=0)), (SHAPE, dict(page=24)), (SHAPE, dict(n_pages=2 ** 27, page=16)),
    (VALUE, dict(qw=G, eps=-1.0)), (VALUE, dict(kw=G, eps=NAN)), (VALUE, dict(kw=G, eps=INF)),
    (ALIGN, dict(q=G + 8)), (ALIGN, dict(qw=G + 2)), (ALIGN, dict(q_out=G + 8)), (ALIGN, dict(pk=G + 8)), (ALIGN, dict(rot_table=G + 8)), (ALIGN, dict(positions=G + 2)),
    (ALIGN, dict(slots=G + 4)), (ALIGN, dict(bits=8, ks=G + 1, vs=G)),
    (OK, dict(M=0)), (OK, dict(M=0, rot=0, rot_table=None, positions=None, n_positions=0)), (OK, dict(M=0, eps=NAN)),
])
def test_append(code, kw):
    assert call(eora.lib.eora_cache_append, APPEND, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(q=None)), (NULL, dict(table=None)), (NULL, dict(lengths=None)), (NULL, dict(out=None)), (NULL, dict(pk=None)), (NULL, dict(pv=None)),
    (NULL, dict(bits=8, vs=G)), (UNSUPPORTED, dict(bits=32)), (UNSUPPORTED, dict(dim=32, q_stride=256)),
    (SHAPE, dict(B=-1)), (SHAPE, dict(B=8193)), (SHAPE, dict(heads=7, q_stride=448)), (SHAPE, dict(heads=0)), (SHAPE, dict(kv=0)), (SHAPE, dict(width=0)),
    (SHAPE, dict(window=-1)), (SHAPE, dict(q_stride=511)), (SHAPE, dict(q_stride=520 + 4)), (SHAPE, dict(page=8)), (SHAPE, dict(width=2 ** 26 + 1)),
    (SHAPE, dict(B=8192, heads=2 ** 12, kv=2 ** 12, q_stride=2 ** 18, width=128)),
    (VALUE, dict(scale=NAN)), (VALUE, dict(scale=-INF)),
    (ALIGN, dict(q=G + 2)), (ALIGN, dict(out=G + 8)), (ALIGN, dict(table=G + 2)), (ALIGN, dict(lengths=G + 1)), (ALIGN, dict(lse=G + 2)), (ALIGN, dict(ws=G + 4)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=eora.cache_attention_workspace_bytes(3, 8, 2, 64, 128) - 1)),
    (OK, dict(B=0)), (OK, dict(B=0, bits=8, ks=G, vs=G)),
])
def test_attention(code, kw):
    assert call(eora.lib.eora_cache_attention, ATTENTION, **kw) == code


def test_workspace_sizes():
    a = eora.adapters_workspace_bytes
    assert a(4, 256, 40, 64) == 0 and a(4, 200, 32, 64) == 0 and a(4, 256, 32, 0) == 0 and a(-1, 256, 32, 64) == 0 and a(4, 256, 32, 1024) == 0
    assert 0 < a(0, 256, 32, 64) <= a(1, 256, 32, 64) <= a(5, 256, 32, 64) <= a(5, 256, 32, 128) <= a(300, 256, 32, 128)
    t = eora.cache_attention_workspace_bytes
    assert t(8193, 8, 2, 64, 128) == 0 and t(3, 7, 2, 64, 128) == 0 and t(3, 8, 2, 96, 128) == 0 and t(3, 8, 2, 64, -1) == 0
    for heads, kv, dim in ((8, 8, 64), (8, 1, 128), (40, 2, 256)):
        assert 0 < t(0, heads, kv, dim, 0) <= t(1, heads, kv, dim, 16) <= t(64, heads, kv, dim, 4096) <= t(8192, heads, kv, dim, 1 << 17)


@pytest.mark.gpu                                         # (the binding asks torch for its stream)
def test_binding_raises_with_the_code():
    with pytest.raises(eora.EoraError) as e:
        eora.linear_adapters(*[None] * 10, 4, 256, 32, 64, 3, 16, None)
    assert e.value.status == NULL and "linear_adapters" in str(e.value)
    with pytest.raises(eora.EoraError) as e:
        eora.cache_attention(*[None] * 9, 3, 8, 2, 64, 512, 4, 16, 16, 8, 0, 0.125, None)
    assert e.value.status == NULL
    with pytest.raises(eora.EoraError) as e:
        eora.cache_append(*[None] * 13, 1, 8, 2, 64, 512, 128, 128, 64, False, 100, 0.0, 4, 16, 16)
    assert e.value.status == NULL
