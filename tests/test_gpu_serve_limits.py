"""What a run of requests refuses, and where it has to go on: windows, room, evictions, decoding past the first table."""
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_14779_amd.serve import ServeRun   # noqa: E402

pytestmark = pytest.mark.gpu

SHAPE = types.SimpleNamespace(layers=1, kv_heads=2, head_dim=64, block_size=16)
HEADS = 8


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture
def make():
    runs = []

    def new_run(contexts, room, **kw):
        runs.append(ServeRun(SHAPE, HEADS, contexts, room, **kw))
        g = torch.Generator(device="cuda").manual_seed(3)
        runs[-1].cache.copy_(torch.randn(runs[-1].cache.shape, generator=g, device="cuda"))
        return runs[-1]
    yield new_run
    for r in runs:
        r.close()


def _step(run, new, seed=0):
    run.begin(new)
    g = torch.Generator(device="cuda").manual_seed(seed)
    return run.layer(0, torch.randn(run.total, HEADS + 4, 64, generator=g, device="cuda").to(torch.bfloat16))


def test_no_eviction_under_a_window(make):
    """A window counts cache indexes: an eviction would leave recent tokens outside it and old ones inside."""
    run = make([300, 77], 64, window=32)
    _step(run, [3, 1])
    before, lens = run.cache.clone(), run.lens.copy()
    with pytest.raises(ValueError, match="window"):
        run.evict(64, recent=8)
    assert torch.equal(run.cache, before) and np.array_equal(run.lens, lens)
    assert torch.isfinite(_step(run, [1, 1])).all()


def test_every_sequence_has_its_own_room(make):
    """200 more tokens are fewer than the longest sequence may have in all, and more than the short one's slots hold."""
    run = make([300, 77], 64)
    for new in ([0, 200], [0, 65], [65, 0]):
        with pytest.raises(ValueError):
            run.begin(new)
        assert run.lens.tolist() == [300, 77] and run.seen.tolist() == [300, 77]
    slot, off = int(run.tables[1][140 // 16]), 140 % 16
    run.cache[0, :, slot, :, off] = 0
    _step(run, [0, 64])
    assert run.lens.tolist() == [300, 141]
    assert run.pos[0, 1, 0, 140].item() == 140 and (run.cache[0, :, slot, :, off] != 0).any(-1).all()   # written
    run.offload()
    run.fetch()


def test_recent_tokens_fit_what_is_kept(make):
    run = make([300, 77], 64)
    _step(run, [3, 1])
    before = run.cache.clone()
    for keep, recent in ((8, 9), (0, 1), (-1, 0), (64, -1)):
        with pytest.raises(ValueError):
            run.evict(keep, recent)
    assert torch.equal(run.cache, before) and run.lens.tolist() == [303, 78]
    run.evict(9, 9)                                    # the last ones and no others
    for s, n in enumerate((303, 78)):
        for h in range(2):
            assert sorted(run.pos[0, s, h, :9].tolist()) == list(range(n - 9, n))


def test_only_what_the_pool_has_is_fetched(make):
    """A request of fewer tokens in as many blocks would overwrite the newer ones."""
    run = make([300, 77], 64)
    with pytest.raises(ValueError):
        run.fetch()                                    # nothing is in the pool yet
    run.offload()
    run.fetch()
    _step(run, [0, 2])                                 # 79 tokens lie in as many blocks as 77
    before = run.cache.clone()
    with pytest.raises(ValueError, match="1"):
        run.fetch()
    assert torch.equal(run.cache, before)
    run.offload()
    run.cache.zero_()
    run.fetch()
    slot = torch.from_numpy(np.repeat(run.tables[1], 16)[:79].astype(np.int64)).cuda()
    off = torch.arange(79, device="cuda") % 16
    assert torch.equal(run.cache[0][:, slot, :, off], before[0][:, slot, :, off])
    run.evict(300, recent=4)                           # nothing to evict
    run.fetch()
    run.evict(299, recent=4)
    with pytest.raises(ValueError, match="0"):
        run.fetch()


def test_sequences_without_tokens(make):
    """A request that has just begun, and one of which eviction left nothing."""
    run = make([0, 77], 64)
    run.offload()
    run.fetch()
    _step(run, [5, 0])
    run.evict(0, recent=0)
    assert run.lens.tolist() == [0, 0]
    run.offload()                                      # the request of 77 tokens is released
    assert run.requests == [None, None]
    run.fetch()
    assert torch.isfinite(_step(run, [1, 2])).all() and run.positions.tolist() == [5, 77, 78]
    run.offload()
    run.fetch()


def test_decoding_goes_on_after_evictions(make):
    """Far past the positions that the first lengths and their room make: each new token is rotated by its own."""
    run = make([300, 77], 32)
    for i in range(12):                                # 300 + 12 * 32 positions
        _step(run, [32, 32 if i % 2 else 0], seed=i)
        run.evict(77, recent=8)
    assert run.seen.tolist() == [684, 269]
    g = torch.Generator(device="cuda").manual_seed(99)
    qkv = torch.randn(2, HEADS + 4, 64, generator=g, device="cuda").to(torch.bfloat16)
    run.begin([1, 1])
    run.layer(0, qkv)
    f = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device="cuda") / 64)
    a = torch.tensor([684.0, 269.0], dtype=torch.float64, device="cuda")[:, None, None] * f
    lo, hi = qkv.double()[:, :HEADS, :32], qkv.double()[:, :HEADS, 32:]
    want = torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)
    # one rounding to bf16, and cosines and sines in 32 bits
    size = torch.cat([lo.abs() + hi.abs()] * 2, -1)
    assert ((run.q.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.001 + 2.0 ** -22 * size).all()
