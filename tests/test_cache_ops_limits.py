"""What the operators on the paged cache take and refuse at the limits that their header names, without a GPU."""
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
