"""A run of requests on a device that is not the current one: its operators are called with its device current."""
import contextlib
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_14779_amd import serve   # noqa: E402


class _Cuda:
    """The current device, without a GPU."""

    def __init__(self):
        self.current = 0

    @contextlib.contextmanager
    def device(self, d):
        before, self.current = self.current, torch.device(d).index
        yield
        self.current = before

    def current_stream(self, d):
        return types.SimpleNamespace(cuda_stream=0)


@pytest.fixture
def run(monkeypatch):
    cuda, called = _Cuda(), []
    for name in ("rope_table", "rope_append", "attention", "attention_mass", "evict"):
        monkeypatch.setattr(serve.K, name, lambda *a, _n=name, **kw: called.append((_n, cuda.current)), raising=False)
    for name in ("attention_workspace", "evict_workspace"):
        monkeypatch.setattr(serve.K, name, lambda *a: 0, raising=False)
    monkeypatch.setattr(serve.K, "Batch", lambda *a: None, raising=False)
    run = object.__new__(serve.ServeRun)
    run.torch = types.SimpleNamespace(cuda=cuda, float32=torch.float32, uint8=torch.uint8, empty_like=torch.empty_like,
                                      empty=lambda *a, device, **kw: torch.empty(*a, **kw))
    run.device, run.dtype = torch.device("cuda", 1), torch.bfloat16
    run._dev = lambda a, dtype=None: torch.as_tensor(np.ascontiguousarray(a, dtype=dtype or np.int32))
    run.shape = types.SimpleNamespace(layers=1, kv_heads=2, head_dim=64, block_size=16)
    run.q_heads, run.n, run.window, run.stride, run.max_kv, run.rope, run.rot = 8, 1, 0, 4, 64, {}, 64
    run.lens, run.seen, run.most = np.array([30], np.int32), np.array([30], np.int64), np.array([64], np.int64)
    run.held, run._work, run.n_positions = np.ones(1, bool), None, 8
    run.table, run.cache_shape, run.k_ptrs, run.v_ptrs = torch.zeros(1, 4, dtype=torch.int32), None, [0], [0]
    run.score, run.pos = torch.zeros(1, 1, 2, 64), torch.zeros(1, 1, 2, 64, dtype=torch.int32)
    return run, called, cuda


def test_operators_run_on_the_run_s_device(run):
    run, called, cuda = run
    run.begin([2])                                     # past the 8 positions: a new table
    run.layer(0, types.SimpleNamespace(shape=(2, 12, 64), dtype=run.dtype, device=run.device, is_contiguous=lambda: True,
                                       data_ptr=lambda: 0x10000))
    run.evict(16, recent=4)
    assert called == [(n, 1) for n in ("rope_table", "rope_append", "attention", "attention_mass", "evict")]
    assert cuda.current == 0


def test_projections_elsewhere_are_refused(run):
    """Their address would be followed by kernels on the run's device."""
    run, called, _ = run
    run.begin([2])
    del called[:]
    with pytest.raises(ValueError, match="cpu"):
        run.layer(0, torch.zeros(2, 12, 64, dtype=torch.bfloat16))
    assert not called
