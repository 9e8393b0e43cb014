"""What the operators on the paged cache take and refuse at the limits that their header names, without a GPU."""
import os

import pytest

from paper_2606_14779_amd import kvpool as K

P = 0x10000         # an aligned address


def _shape(heads=8, kv_heads=2, head_dim=64, block=16, slots=100):
    return K.CacheShape("bf16", heads, kv_heads, head_dim, block, slots)


@pytest.mark.parametrize("sizes", [(1, 1, 1, 131072), (2, 4, 3, 640), (1, 512, 512, 131072), (9, 0, 0, 20000), (0, 0, 0, 0)])
def test_workspaces_are_asked_for_by_sizes_alone(sizes):
    """Before the batch's arrays exist, and the same as with them."""
    n_seq, total, max_q, max_kv = sizes
    there = K.Batch(n_seq, total, max_q, max_kv, P, P, P, 8192)
    absent = K.Batch(n_seq, total, max_q, max_kv, 0, 0, 0, 0)
    for f in (K.attention_workspace, K.evict_workspace):
        assert f(_shape(), absent) == f(_shape(), there)
    assert K.evict_workspace(_shape(), K.Batch(n_seq, 0, 0, max_kv, 0, 0, 0, 0)) == K.evict_workspace(_shape(), there)


def _refused(f, *a, **kw):
    with pytest.raises(K.KVPoolError) as e:
        f(*a, **kw)
    assert e.value.name == "INVALID"
    return str(e.value)


def test_limits_of_single_calls_are_those_of_the_header():
    one = _shape(heads=1, kv_heads=1)
    most = K.Batch(1, 1 << 24, 1, 16, P, P, P, 1)      # as many new tokens as every other call takes
    assert "2^24" in _refused(K.rope_append, one, most, P, 100, 64, P, P, 64, P, 64, P, P)
    K.attention_workspace(one, most)
    for n_seq, heads, max_kv in ((1 << 11, 8, 131072), (1 << 18, 1, 8192), (1, 2, 1 << 30)):
        tokens = K.Batch(n_seq, 0, 0, max_kv, P, P, P, (1 << 30) // 16)
        shape = _shape(heads=heads, kv_heads=heads)
        _refused(K.attention_mass, shape, tokens, 0, 64, P, 1.0, 0, 0, P, max_kv)
        K.evict_workspace(shape, tokens)
    with open(os.path.join(os.path.dirname(__file__), "..", "include", "kvpool.h")) as f:
        header = f.read()
    for words in ("kv_rope_append takes less than 2^24 new tokens", "2^24 of n_seq * num_kv_heads * ceil(max_kv / 128)"):
        assert words in " ".join(header.replace("\n *", " ").split())
