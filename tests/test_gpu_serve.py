"""The operators together with the pool: a request fetched, extended, evicted and offloaded again."""
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_14779_amd.serve import ServeRun   # noqa: E402

pytestmark = pytest.mark.gpu

SHAPE = types.SimpleNamespace(layers=2, kv_heads=2, head_dim=64, block_size=16)


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _tokens(run, layer, kv, s, head, n):
    slot = torch.from_numpy(np.repeat(run.tables[s], 16)[:n].astype(np.int64)).cuda()
    return run.cache[layer, kv][slot, head, torch.arange(n, device="cuda") % 16].double()


def _rotated(x, positions, base):
    """[tokens][heads][64] by their positions, in 64 bits."""
    f = base ** (-torch.arange(0, 64, 2, dtype=torch.float64, device="cuda") / 64)
    a = positions.double()[:, None, None] * f
    lo, hi = x.double()[..., :32], x.double()[..., 32:]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


def test_round_trip():
    contexts, heads, new = [300, 77], 8, [20, 5]
    run = ServeRun(SHAPE, heads, contexts, room=64, rope=dict(base=10000.0))
    g = torch.Generator(device="cuda").manual_seed(1)
    run.cache.copy_(torch.randn(run.cache.shape, generator=g, device="cuda"))
    before = [_tokens(run, 1, 0, s, 1, n) for s, n in enumerate(contexts)]
    run.offload()
    run.cache.fill_(float("nan"))
    run.fetch()
    for s, n in enumerate(contexts):
        assert torch.equal(_tokens(run, 1, 0, s, 1, n), before[s])
    run.begin(new)
    qkv = [torch.randn(25, heads + 4, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    outs = [run.layer(i, x) for i, x in enumerate(qkv)]
    for i in range(2):
        # keys and queries as rotated in 64 bits and rounded: a unit in the last place each
        q = _rotated(qkv[i][:, :heads], run.positions, 10000.0)
        assert (run.q.double() - q).abs().max().item() <= 2.0 ** -8 * q.abs().max().item() if i == 1 else True
        for s, (c, k) in enumerate(zip(contexts, new)):
            rows = slice(0, 20) if s == 0 else slice(20, 25)
            for h in range(heads):
                keys, values = (_tokens(run, i, kv, s, h // 4, c + k) for kv in (0, 1))
                rotated = _rotated(qkv[i][rows, heads + h // 4, None], run.positions[rows], 10000.0)[:, 0]
                assert ((keys[c:] - rotated).abs() <= 2.0 ** -8 * rotated.abs() + 1e-5).all()
                assert torch.equal(values[c:], qkv[i][rows, heads + 2 + h // 4].double())
                z = q[rows, h].to(torch.bfloat16).double() @ keys.t().contiguous() / 8.0
                z = z.masked_fill(torch.arange(c + k, device="cuda")[None] > torch.arange(c, c + k, device="cuda")[:, None],
                                  -np.inf)
                want = torch.softmax(z, -1) @ values
                # a query that rounds the other way moves logits by up to 2^-8 |q| |k|: a few hundredths in all
                assert (outs[i][rows, h].double() - want).abs().max().item() < 0.05
    weight = run.score[1].double().sum(-1)
    assert torch.allclose(weight, torch.tensor([[80.0, 80.0], [20.0, 20.0]], dtype=torch.float64, device="cuda"), rtol=1e-4)
    kept = {}
    for s, (c, k) in enumerate(zip(contexts, new)):
        score = run.score[1, s, 1, :c + k].cpu().numpy()
        best = np.lexsort((np.arange(c + k), -score, np.arange(c + k) < c + k - 8))[:64]
        kept[s] = {int(p): _tokens(run, 1, 0, s, 1, c + k)[p] for p in best}
    run.evict(64, recent=8)
    assert run.lens.tolist() == [64, 64]
    run.offload()                                          # the smaller request replaces the first one
    run.cache.zero_()
    run.fetch()
    for s in range(2):
        keys, pos = _tokens(run, 1, 0, s, 1, 64), run.pos[1, s, 1, :64].tolist()
        assert set(pos) == set(kept[s])
        for at, p in enumerate(pos):
            assert torch.equal(keys[at], kept[s][p])
    run.begin([1, 1])
    assert run.positions.tolist() == [320, 82]
    out = run.layer(0, torch.randn(2, heads + 4, 64, generator=g, device="cuda").to(torch.bfloat16))
    assert torch.isfinite(out).all()
    with pytest.raises(ValueError):
        run.begin([1000, 0])
    run.close()
