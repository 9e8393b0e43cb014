"""What the operators on the paged cache refuse, before any GPU call (the pointers here are never followed), and
what they say about their workspaces."""
import math

import pytest

from paper_2606_14779_amd import kvpool as K

P = 0x10000         # an aligned address


def _shape(dtype="bf16", heads=8, kv_heads=2, head_dim=64, block=16, slots=100):
    return K.CacheShape(dtype, heads, kv_heads, head_dim, block, slots)


def _batch(n_seq=2, total=4, max_q=3, max_kv=640, cu=P, kv_len=P, table=P, stride=40):
    return K.Batch(n_seq, total, max_q, max_kv, cu, kv_len, table, stride)


def _attention(shape=None, batch=None, q=P, q_stride=512, k=P, v=P, scale=1.0, out=P, out_stride=512, **kw):
    K.attention(shape or _shape(), batch or _batch(), q, q_stride, k, v, scale, out, out_stride,
                **dict(dict(workspace=P, workspace_bytes=1 << 40), **kw))


def _mass(shape=None, batch=None, q=P, q_stride=512, k=P, scale=1.0, lse=P, score_in=0, score_out=P, stride=640, **kw):
    K.attention_mass(shape or _shape(), batch or _batch(), q, q_stride, k, scale, lse, score_in, score_out, stride, **kw)


def _evict(shape=None, batch=None, keep=P, score_in=P, score_out=P, stride=640, k=P, v=P, len_out=P, work=P, n=1 << 40, **kw):
    K.evict(shape or _shape(), batch or _batch(), keep, score_in, score_out, stride, k, v, len_out, work, n, **kw)


def _rope(shape=None, batch=None, table=P, n=100, rot=64, positions=P, k=P, k_stride=128, v=P, v_stride=128, kc=P, vc=P, **kw):
    K.rope_append(shape or _shape(), batch or _batch(), table, n, rot, positions, k, k_stride, v, v_stride, kc, vc, **kw)


def _refused(f, *a, **kw):
    with pytest.raises(K.KVPoolError) as e:
        f(*a, **kw)
    assert e.value.name == "INVALID"
    return str(e.value)


SHAPES = [dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264),
          dict(block=0), dict(slots=0), dict(slots=1 << 31), dict(heads=1 << 17), dict(block=1 << 17)]
BATCHES = [dict(max_kv=641), dict(max_q=5), dict(kv_len=0), dict(kv_len=P + 2), dict(table=0), dict(table=P + 1),
           dict(max_kv=(1 << 30) + 1, stride=1 << 30), dict(n_seq=1 << 22), dict(n_seq=(1 << 17) + 1)]


@pytest.mark.parametrize("call", [_attention, _mass, _evict, _rope])
@pytest.mark.parametrize("bad", SHAPES, ids=str)
def test_shapes_refused(call, bad):
    _refused(call, shape=_shape(**bad))


@pytest.mark.parametrize("call", [_attention, _mass, _evict, _rope])
@pytest.mark.parametrize("bad", BATCHES, ids=str)
def test_batches_refused(call, bad):
    if call is _evict and "max_q" in bad:
        pytest.skip("eviction looks at no queries")
    _refused(call, batch=_batch(**bad))


@pytest.mark.parametrize("call", [_attention, _mass, _rope])
def test_queries_refused(call):
    _refused(call, batch=_batch(cu=0))
    _refused(call, batch=_batch(n_seq=0))
    _refused(call, batch=_batch(total=1 << 28))


@pytest.mark.parametrize("bad", [dict(q=0), dict(q=P + 8), dict(q_stride=513), dict(k=0), dict(v=P + 2), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(out=0), dict(out_stride=504),
                                 dict(sinks=P + 2), dict(lse=P + 1), dict(workspace=0), dict(workspace=P + 8),
                                 dict(workspace_bytes=8), dict(q_stride=(1 << 40) + 8)], ids=str)
def test_attention_refuses(bad):
    _refused(_attention, **bad)


@pytest.mark.parametrize("bad", [dict(q=0), dict(q_stride=4), dict(k=0), dict(scale=0.0), dict(lse=0), dict(lse=P + 2),
                                 dict(score_in=P + 2), dict(score_out=0), dict(stride=639)], ids=str)
def test_mass_refuses(bad):
    _refused(_mass, **bad)


@pytest.mark.parametrize("bad", [dict(keep=0), dict(keep=P + 2), dict(score_in=0), dict(score_out=0), dict(stride=639),
                                 dict(k=0), dict(v=P + 8), dict(len_out=0), dict(work=0), dict(work=P + 8), dict(n=100),
                                 dict(protect=P + 1), dict(pos_in=P + 2, pos_stride=640), dict(pos_in=P, pos_stride=639),
                                 dict(pos_out=P)], ids=str)
def test_evict_refuses(bad):
    _refused(_evict, **bad)


@pytest.mark.parametrize("bad", [dict(table=0), dict(table=P + 4), dict(n=0), dict(rot=63), dict(rot=66), dict(positions=0),
                                 dict(k=0), dict(k_stride=129), dict(v=P + 8), dict(kc=0), dict(vc=P + 2), dict(q=P),
                                 dict(q_out=P), dict(q=P, q_out=P, q_stride=512, q_out_stride=512),
                                 dict(q=P, q_out=2 * P, q_stride=512, q_out_stride=504), dict(pos=P, pos_stride=639),
                                 dict(pos=P + 2, pos_stride=640)], ids=str)
def test_rope_append_refuses(bad):
    _refused(_rope, **bad)


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=3), dict(rot=258), dict(base=0.0), dict(base=math.nan),
                                 dict(magnitude=0.0), dict(kind="linear", factor=0.5), dict(table=0), dict(table=P + 4),
                                 dict(kind="by_parts", factor=2.0), dict(n=(1 << 30) + 1),
                                 dict(kind="by_parts", factor=2.0, original_length=10.0, alpha=4.0, beta=4.0),
                                 dict(kind="by_parts_index", factor=2.0, original_length=10.0, alpha=1.0, beta=4.0, base=1.0)],
                         ids=str)
def test_rope_table_refuses(bad):
    a = dict(dict(table=P, n=10, rot=64), **bad)
    _refused(K.rope_table, a.pop("table"), a.pop("n"), a.pop("rot"), **a)


def test_python_side_refusals():
    with pytest.raises(ValueError):
        _shape(dtype="f32")
    with pytest.raises(ValueError):
        _shape(heads=-1)
    with pytest.raises(ValueError):
        _batch(total=1 << 32)
    with pytest.raises(ValueError):
        _attention(window=-1)
    with pytest.raises(ValueError):
        _mass(last=-1)
    with pytest.raises(ValueError):
        K.rope_table(P, 10, 64, kind="other")
    for bad in (dict(q_stride=-8), dict(out_stride=1 << 64), dict(workspace_bytes=-1), dict(window=1 << 32)):
        with pytest.raises(ValueError):
            _attention(**bad)
    for bad in (dict(q_stride=1 << 64), dict(last=1 << 32), dict(stride=-1)):
        with pytest.raises(ValueError):
            _mass(**bad)
    for bad in (dict(stride=-1), dict(pos_stride=1 << 32), dict(n=-1)):
        with pytest.raises(ValueError):
            _evict(**bad)
    for bad in (dict(n=-1), dict(rot=1 << 32), dict(pos_stride=-1), dict(k_stride=-8), dict(v_stride=1 << 64),
                dict(q_stride=-8), dict(q_out_stride=1 << 65)):
        with pytest.raises(ValueError):
            _rope(**bad)


def test_null_structures_and_reserved_fields():
    lib, shape, batch = K._lib, _shape(), _batch()
    for f in (lib.kv_attention_workspace, lib.kv_evict_workspace):
        assert f(None, batch._p, P) == -1 and f(shape._p, None, P) == -1 and f(shape._p, batch._p, None) == -1
    assert lib.kv_rope_table(P, 10, 64, None, None) == -1
    for s, field in ((_shape(), "reserved"), (_shape(), "dtype")):
        setattr(s._c, field, 5)
        _refused(K.attention_workspace, s, batch)
    batch._c.reserved = 1
    _refused(K.evict_workspace, shape, batch)


def test_workspaces():
    """None where the keys are not split, bounded by a few parts of the output where they are."""
    assert K.attention_workspace(_shape(), _batch(max_kv=16)) == 0
    assert K.attention_workspace(_shape(), _batch(n_seq=0, total=0, max_q=0)) == 0
    for total, max_q, kv in ((1, 1, 131072), (512, 512, 131072), (7, 3, 5000), (4096, 4096, 4096)):
        n = K.attention_workspace(_shape(), _batch(n_seq=1, total=total, max_q=max_q, max_kv=kv, stride=8192))
        part = total * 8 * (64 + 2) * 4
        assert n % part == 0 and n // part <= 1024 and (n // part) * 128 <= max(kv, 128) + 127
    assert K.evict_workspace(_shape(), _batch()) >= 2 * 2 * 640 // 2 * 8
