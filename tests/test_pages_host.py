"""What the operators on pages of either kind and on drafted tokens refuse, before any GPU call (the pointers here are
never followed), and what they say about pages and workspaces."""
import math

import pytest

from paper_2606_14779_amd import kvpool as K
from test_cache_ops_host import BATCHES, P, SHAPES, _batch, _refused, _shape


def _pages(kind="e4m3", k=P, v=P):
    return K.Pages(kind, k, v)


def _attend(shape=None, batch=None, pages=None, q=P, q_stride=512, scale=1.0, out=P, out_stride=512, **kw):
    K.attention_pages(shape or _shape(), batch or _batch(), pages or _pages(), q, q_stride, scale, out, out_stride,
                      **dict(dict(workspace=P, workspace_bytes=1 << 40), **kw))


def _append(shape=None, batch=None, pages=None, table=P, n=100, rot=64, positions=P, k=P, k_stride=128, v=P, v_stride=128,
            **kw):
    K.norm_rope_append(shape or _shape(), batch or _batch(), pages or _pages(), table, n, rot, positions, k, k_stride, v,
                       v_stride, **kw)


def _convert(shape=None, batch=None, pages=None, to=None, table=P, stride=40, slots=100, **kw):
    K.convert_pages(shape or _shape(), batch or _batch(), pages or _pages(), to or _pages("16"), table, stride, slots, **kw)


def _commit(shape=None, batch=None, pages=None, path=P, accepted=P, len_out=2 * P, **kw):
    K.tree_commit(shape or _shape(), batch or _batch(), pages or _pages(), path, accepted, len_out, **kw)


CALLS = [_attend, _append, _convert, _commit]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad", SHAPES, ids=str)
def test_shapes_refused(call, bad):
    _refused(call, shape=_shape(**bad))


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("bad", BATCHES, ids=str)
def test_batches_refused(call, bad):
    if call is _convert and "max_q" in bad:
        pytest.skip("a conversion looks at no queries")
    _refused(call, batch=_batch(**bad))


@pytest.mark.parametrize("call", [_attend, _append, _commit])
def test_queries_refused(call):
    _refused(call, batch=_batch(cu=0))
    _refused(call, batch=_batch(n_seq=0))
    _refused(call, batch=_batch(total=1 << 28))


@pytest.mark.parametrize("call", CALLS)
def test_pages_refused(call):
    for bad in (dict(k=0), dict(v=0), dict(k=P + 8), dict(v=P + 2)):
        _refused(call, pages=_pages(**bad))
    for field, value in (("kind", 2), ("reserved", 1)):
        p = _pages()
        setattr(p._c, field, value)
        _refused(call, pages=p)
    _refused(call, shape=_shape(heads=128, kv_heads=128, head_dim=256, block=65536, slots=1))   # elements of a slot


@pytest.mark.parametrize("bad", [dict(q=0), dict(q=P + 8), dict(q_stride=513), dict(scale=0.0), dict(scale=-1.0),
                                 dict(scale=math.nan), dict(scale=math.inf), dict(out=0), dict(out_stride=504),
                                 dict(sinks=P + 2), dict(lse=P + 1), dict(workspace=0), dict(workspace=P + 8),
                                 dict(workspace_bytes=8), dict(q_stride=(1 << 40) + 8), dict(tree=P + 4, tree_words=1),
                                 dict(tree=P, tree_words=0), dict(tree=0, tree_words=1), dict(tree=P, tree_words=(1 << 20) + 1)],
                         ids=str)
def test_attention_pages_refuses(bad):
    _refused(_attend, **bad)


def test_a_tree_of_too_few_words():
    _refused(_attend, batch=_batch(total=70, max_q=65), tree=P, tree_words=1)


@pytest.mark.parametrize("bad", [dict(table=0), dict(table=P + 4), dict(n=0), dict(rot=63), dict(rot=66), dict(positions=0),
                                 dict(k=0), dict(k_stride=129), dict(v=P + 8), dict(q=P), dict(q_out=P),
                                 dict(q=P, q_out=P, q_stride=512, q_out_stride=512),
                                 dict(q=P, q_out=2 * P, q_stride=512, q_out_stride=504), dict(pos=P, pos_stride=639),
                                 dict(pos=P + 2, pos_stride=640), dict(norm=K.HeadNorm(P + 8, P, 1e-6)),
                                 dict(norm=K.HeadNorm(P, P + 2, 1e-6)), dict(norm=K.HeadNorm(P, P, -1e-6)),
                                 dict(norm=K.HeadNorm(P, P, math.nan)), dict(norm=K.HeadNorm(P, P, math.inf)),
                                 dict(axes=K.RopeAxes(0, [0] * 32)), dict(axes=K.RopeAxes(5, [0] * 32)),
                                 dict(axes=K.RopeAxes(2, [0] * 31 + [2]))], ids=str)
def test_norm_rope_append_refuses(bad):
    _refused(_append, **bad)


def test_reserved_fields_of_norm_and_axes():
    for name, x in (("norm", K.HeadNorm(P, P, 0.0)), ("axes", K.RopeAxes(1, [0] * 32))):
        x._c.reserved = 1
        _refused(_append, **{name: x})


def test_convert_pages_refuses():
    for bad in (dict(table=0), dict(table=P + 2), dict(stride=39), dict(slots=0), dict(slots=1 << 30), dict(first=P + 1),
                dict(to=_pages()), dict(pages=_pages("16")), dict(to=_pages("16", k=0)), dict(to=_pages("16", v=P + 8))):
        _refused(_convert, **bad)
    _refused(_convert, shape=_shape(heads=64, kv_heads=64, slots=1), batch=_batch(n_seq=4096, max_kv=1 << 20, stride=1 << 16),
             stride=1 << 16)


@pytest.mark.parametrize("bad", [dict(path=0), dict(path=P + 2), dict(accepted=0), dict(accepted=P + 1), dict(len_out=0),
                                 dict(len_out=P + 2), dict(pos=P, pos_stride=639), dict(pos=P + 2, pos_stride=640)], ids=str)
def test_tree_commit_refuses(bad):
    _refused(_commit, **bad)


def test_python_side_refusals():
    for bad in (dict(kind="e5m2"), dict(k=-1), dict(v=1 << 64)):
        with pytest.raises(ValueError):
            _pages(**bad)
    with pytest.raises(ValueError):
        K.page_bytes(_shape(), "8")
    with pytest.raises(ValueError):
        K.HeadNorm(-1, 0, 0.0)
    for bad in ((1, [0] * 129), (1, [256]), (1, [-1]), (-1, [0])):
        with pytest.raises(ValueError):
            K.RopeAxes(*bad)
    with pytest.raises(ValueError):
        _append(axes=K.RopeAxes(1, [0] * 31))
    for bad in (dict(q_stride=-8), dict(out_stride=1 << 64), dict(workspace_bytes=-1), dict(window=1 << 32),
                dict(tree_words=-1)):
        with pytest.raises(ValueError):
            _attend(**bad)
    for bad in (dict(n=-1), dict(rot=1 << 32), dict(pos_stride=-1), dict(k_stride=-8), dict(v_stride=1 << 64),
                dict(q_stride=-8), dict(q_out_stride=1 << 65)):
        with pytest.raises(ValueError):
            _append(**bad)
    for bad in (dict(stride=-1), dict(slots=1 << 32)):
        with pytest.raises(ValueError):
            _convert(**bad)
    with pytest.raises(ValueError):
        _commit(pos_stride=1 << 32)


def test_null_structures():
    lib, shape, batch, pages = K._lib, _shape(), _batch(), _pages()
    assert lib.kv_attention_pages_workspace(None, batch._p, P) == -1
    assert lib.kv_attention_pages_workspace(shape._p, None, P) == -1
    assert lib.kv_attention_pages_workspace(shape._p, batch._p, None) == -1
    assert lib.kv_page_bytes(None, 0, P) == -1 and lib.kv_page_bytes(shape._p, 0, None) == -1
    assert lib.kv_page_bytes(shape._p, 2, P) == -1
    assert lib.kv_attention_pages(shape._p, batch._p, None, None, 0, P, 512, 1.0, 0, None, P, 512, None, P, 1 << 40, None) == -1
    assert lib.kv_tree_commit(shape._p, batch._p, None, P, P, None, 0, P, None) == -1
    assert lib.kv_convert_pages(shape._p, batch._p, pages._p, None, P, 40, 100, None, None) == -1
    assert lib.kv_convert_pages(shape._p, batch._p, None, pages._p, P, 40, 100, None, None) == -1


def test_empty_batches_look_at_no_buffers():
    none = dict(batch=_batch(n_seq=0, total=0, max_q=0, max_kv=0, cu=0, kv_len=0, table=0), pages=_pages(k=0, v=0))
    _attend(**none, q=0, out=0)
    _append(**none, positions=0, k=0, v=0)
    _convert(**none, to=_pages("16", 0, 0), table=0)
    _commit(**none, path=0, accepted=0, len_out=0)


@pytest.mark.parametrize("d,kv_heads,block,want", [(64, 2, 16, 2 * 16 * 68), (128, 8, 16, 8 * 16 * 132), (8, 1, 1, 16),
                                                   (24, 1, 1, 32), (136, 1, 2, 288), (256, 4, 16, 4 * 16 * 264)])
def test_page_bytes(d, kv_heads, block, want):
    shape = _shape(heads=kv_heads, kv_heads=kv_heads, head_dim=d, block=block)
    assert K.page_bytes(shape, "e4m3") == want and want % 16 == 0
    assert K.page_bytes(shape, "16") == kv_heads * block * d * 2


def test_workspaces():
    """At least that of attention over 16-bit pages, which takes the same calls; bounded by a few parts of the output."""
    assert K.attention_pages_workspace(_shape(), _batch(max_kv=16)) == 0
    assert K.attention_pages_workspace(_shape(), _batch(n_seq=0, total=0, max_q=0)) == 0
    for total, max_q, kv in ((1, 1, 131072), (512, 512, 131072), (7, 3, 5000), (16, 16, 131072), (32, 32, 70000)):
        b = _batch(n_seq=1, total=total, max_q=max_q, max_kv=kv, stride=8192)
        n = K.attention_pages_workspace(_shape(), b)
        part = total * 8 * (64 + 2) * 4
        assert n >= K.attention_workspace(_shape(), b)
        assert n % part == 0 and n // part <= 1024 and (n // part) * 128 <= max(kv, 128) + 127


@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_a_large_windowed_tree_is_cut_by_all_its_drafts(kind):
    """Every row tile goes over the window and all of 2048 drafts, whatever its own rows are: 64 workgroups of 2200 keys
    are cut, and that needs a workspace."""
    shape, batch = _shape(heads=8, kv_heads=1, head_dim=128, slots=1 << 16), _batch(n_seq=1, total=2048, max_q=2048,
                                                                                      max_kv=8192, stride=512)
    tree = dict(shape=shape, batch=batch, pages=_pages(kind), q_stride=1024, out_stride=1024, tree=P, tree_words=32, window=128)
    assert "workspace" in _refused(_attend, **tree, workspace=0)
    need = K.attention_pages_workspace(shape, batch)
    assert "workspace" in _refused(_attend, **tree, workspace_bytes=need // 8)


def test_loads_of_16_elements_stay_in_a_slot():
    """Rows of 8-bit pages are read 16 elements at a time, the last ones of a head of 8 n elements with 8 bytes past it."""
    for d in range(8, 264, 8):
        for rows in range(1, 40):
            shape = _shape(heads=1, kv_heads=1, head_dim=d, block=rows)
            assert (rows - 1) * d + (d + 15) // 16 * 16 <= K.page_bytes(shape, "e4m3")
