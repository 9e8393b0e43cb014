"""What a run with drafted tokens hands to the operators and what it refuses, without a GPU."""
import contextlib
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_14779_amd import drafts   # noqa: E402
from paper_2606_14779_amd.drafts import DraftRun, tree_mask   # noqa: E402

SEEN = [30, 7]


@pytest.fixture
def make(monkeypatch):
    """Runs of two sequences of 30 and 7 cached tokens, whose calls of operators are listed in `called`."""
    def new_run(window=0):
        called = []
        for name in ("norm_rope_append", "attention_pages", "tree_commit"):
            monkeypatch.setattr(drafts.K, name, lambda *a, _n=name, **kw: called.append((_n, a, kw)))
        monkeypatch.setattr(drafts.K, "attention_pages_workspace", lambda *a: 0)
        monkeypatch.setattr(drafts.K, "Batch", lambda *a: a)
        run = object.__new__(DraftRun)
        cuda = types.SimpleNamespace(device=lambda d: contextlib.nullcontext(),
                                     current_stream=lambda d: types.SimpleNamespace(cuda_stream=0))
        run.torch = types.SimpleNamespace(cuda=cuda, float32=torch.float32, uint8=torch.uint8, empty_like=torch.empty_like,
                                          empty=torch.empty, as_tensor=torch.as_tensor)
        run.device, run.dtype = torch.device("cpu"), torch.bfloat16
        run.shape = types.SimpleNamespace(layers=1, kv_heads=2, head_dim=64, block_size=16)
        run.q_heads, run.n, run.window, run.stride, run.max_kv, run.rot = 8, 2, window, 16, 256, 64
        run.lens, run.seen, run.most = np.array(SEEN, np.int32), np.array(SEEN, np.int64), np.array([256, 256], np.int64)
        run.held, run._work, run.n_positions, run.angles = np.ones(2, bool), None, 512, torch.zeros(1)
        run.table, run.cache_shape, run.pages, run.norm = torch.zeros(2, 16, dtype=torch.int32), None, [None], None
        run.pos, run.drafted, run.kind = torch.zeros(1, 2, 2, 256, dtype=torch.int32), None, "e4m3"
        return run, called
    return new_run


def _bits(tree, n):
    return np.unpackbits(tree.numpy().view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)


def _tree(rng, n, back=4):
    return [-1] + [int(rng.integers(max(0, i - back), i)) for i in range(1, n)]


def _ancestors(parents, i):
    """Draft i and those above it, nearest first."""
    out = []
    while i >= 0:
        out.append(i)
        i = parents[i]
    return out


# ---- a window reaches over the drafts

@pytest.mark.parametrize("window", [0, 1, 4, 9, 63, 64, 65, 200])
def test_a_draft_sees_its_window_of_drafts(make, window):
    """The nearest `window` of a draft and its ancestors, in one word or two; places go by all ancestors."""
    rng = np.random.default_rng(window)
    for parents in ([list(range(-1, 9)), [-1, 0, 0]], [_tree(rng, 100), _tree(rng, 20)], [[-1], list(range(-1, 129))]):
        run, _ = make(window)
        new = [len(p) for p in parents]
        words = -(-max(new) // 64)
        masks = [tree_mask(p) for p in parents]
        run.begin(new, np.concatenate([np.pad(m, ((0, 0), (0, words - m.shape[1]))) for m in masks]))
        got, places = _bits(run.tree, max(new)), run.positions.tolist()
        for s, p in enumerate(parents):
            for i in range(new[s]):
                above = _ancestors(p, i)
                want = np.zeros(max(new), bool)
                want[above[:window or None]] = True
                assert (got[sum(new[:s]) + i, :new[s]] == want[:new[s]]).all()
                assert places[sum(new[:s]) + i] == SEEN[s] + len(above) - 1


def test_masks_that_a_window_cannot_place(make):
    """A draft that sees far ones and not those between: what it sees after the far ones are gone does not tell its place.
    Drafts that all see each other stand at one place."""
    far = np.zeros((12, 64), bool)
    np.fill_diagonal(far, True)
    far[11, :11] = True                              # 11 drafts of place 0: 11 places behind them all
    rows = np.packbits(far, axis=1, bitorder="little").view(np.int64)
    run, _ = make(4)
    with pytest.raises(ValueError, match="window"):
        run.begin([12, 0], rows)
    assert run.lens.tolist() == SEEN and run.drafted is None
    run, _ = make(12)
    run.begin([12, 0], rows)
    run, _ = make(2)
    both = np.zeros((6, 64), bool)
    both[:, :5] = True
    both[5, 5] = True
    run.begin([6, 0], np.packbits(both, axis=1, bitorder="little").view(np.int64))
    assert (_bits(run.tree, 6) == both[:, :6]).all() and run.positions.tolist() == [34] * 5 + [35]


# ---- what is committed is a path

def test_only_paths_are_committed(make):
    """One left out would leave a hole in the positions, one of another branch a token that followed others."""
    #            0
    #        1       2
    #      3   4     5
    #          6
    parents = [-1, 0, 0, 1, 1, 2, 4]
    for window in (0, 2):
        for bad in ([1], [0, 3], [0, 1, 2], [0, 1, 3, 4], [0, 1, 6], [0, 4, 6], [6], [0, 1, 5], [0, 2, 6]):
            run, called = make(window)
            run.begin([7, 1], np.concatenate([tree_mask(parents), tree_mask([-1])]))
            with pytest.raises(ValueError, match="path"):
                run.commit([bad, [0]])
            assert not called and run.drafted.tolist() == [7, 1] and run.lens.tolist() == [37, 8]
        for good in ([], [0], [0, 1], [0, 2, 5], [0, 1, 4, 6]):
            run, called = make(window)
            run.begin([7, 1], np.concatenate([tree_mask(parents), tree_mask([-1])]))
            run.commit([good, []])
            assert [c[0] for c in called] == ["tree_commit"] and run.lens.tolist() == [30 + len(good), 7]


def test_two_trees_of_one_sequence(make):
    """Drafts without a parent: each begins a path of its own."""
    for bad in ([0, 1], [1, 2], [0, 3], [0, 1, 2, 3]):
        run, _ = make()
        run.begin([4, 0], tree_mask([-1, -1, 0, 1]))
        with pytest.raises(ValueError, match="path"):
            run.commit([bad, []])
    for good in ([0, 2], [1, 3], [1]):
        run, _ = make()
        run.begin([4, 0], tree_mask([-1, -1, 0, 1]))
        run.commit([good, []])
        assert run.seen.tolist() == [30 + len(good), 7]


def test_drafts_that_see_each_other_are_committed_together(make):
    both = np.zeros((6, 64), bool)
    both[:, :5] = True
    both[5, 5] = True
    rows = np.packbits(both, axis=1, bitorder="little").view(np.int64)
    for paths, ok in (([0, 1], False), ([0, 1, 2, 3, 4], True), ([5], False), ([0, 1, 2, 3, 4, 5], True)):
        run, _ = make()
        run.begin([6, 0], rows)
        with contextlib.nullcontext() if ok else pytest.raises(ValueError, match="path"):
            run.commit([paths, []])


# ---- steps

def _qkv(run):
    return torch.zeros(run.total, 12, 64, dtype=torch.bfloat16)


def test_no_layers_between_commit_and_the_next_step(make):
    """The batch of the step before has lengths that are no longer those of the cache, in memory that may be others'."""
    run, called = make()
    run.begin([2, 1], np.concatenate([tree_mask([-1, 0]), tree_mask([-1])]))
    run.layer(0, _qkv(run))
    run.commit([[0], [0]])
    del called[:]
    with pytest.raises(ValueError, match="step"):
        run.layer(0, _qkv(run))
    assert not called
    run.begin([1, 1])
    run.layer(0, _qkv(run))
    assert [c[0] for c in called] == ["norm_rope_append", "attention_pages"]


def test_a_drafted_step_without_tokens(make):
    """A mask of no rows has no address: no mask, as words of none are refused."""
    for window in (0, 4):
        run, called = make(window)
        run.begin([0, 0], np.zeros((0, 1), np.int64))
        run.layer(0, _qkv(run))
        assert (called[-1][2]["tree"], called[-1][2]["tree_words"]) == (0, 0)
        run.commit([[], []])
        assert run.lens.tolist() == SEEN
