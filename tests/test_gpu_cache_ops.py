"""The operators on the paged cache (rotary append, attention, attention mass, eviction) against plain forms in
64 bits, where they can go wrong: empty rows, sequences without tokens, absent slots, NaN in what is masked, odd
head counts, sizes and strides, short and long lengths, tables of more than 2^32 bytes, graphs and other streams."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_ops_ref as R   # noqa: E402
from paper_2606_14779_amd import kvpool as K   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def run_attention(c, q, scale, window=0, sinks=None, want_lse=True, out=None):
    out = torch.full((c.total, c.heads, c.head_dim), 7.0, dtype=R.DTYPE[c.dtype], device="cuda") if out is None else out
    lse = torch.full((c.heads, c.total), 7.0, dtype=torch.float32, device="cuda") if want_lse else None
    w, n = c.workspace(K.attention_workspace)
    K.attention(c.shape, c.batch, q.data_ptr(), q.stride(0), c.k_cache.data_ptr(), c.v_cache.data_ptr(), scale,
                out.data_ptr(), out.stride(0), window=window, sinks=sinks.data_ptr() if sinks is not None else 0,
                lse=lse.data_ptr() if want_lse else 0, workspace=w.data_ptr(), workspace_bytes=n, stream=_stream())
    return out, lse


def check_attention(c, window=0, with_sinks=False, q=None, scale=None):
    q = c.normal(c.total, c.heads, c.head_dim, std=2.0) if q is None else q
    scale = c.head_dim ** -0.5 if scale is None else scale
    sinks = c.normal(c.heads, std=2.0, to=torch.float32) if with_sinks else None
    out, lse = run_attention(c, q, scale, window, sinks)
    want, want_lse, tol, tol_lse = R.attention(c, q, scale, window, sinks)
    assert torch.isfinite(out).all()
    off = (out.double() - want).abs() - tol
    assert off.max().item() <= 0 if off.numel() else True, "out is off by %g more than it may" % off.max().item()
    same = (lse.double() == want_lse) | ((lse.double() - want_lse).abs() <= tol_lse)
    assert same.all(), "lse is off by %g" % (lse.double() - want_lse).abs()[~same].max().item()
    return q, out, lse


# (new, cached) of every sequence
FEW = {"one": [(1, 1)], "single": [(1, 700)], "ragged": [(1, 1), (1, 2), (1, 33), (1, 129), (1, 1300)],
       "short": [(2, 40), (1, 5), (3, 3)], "gaps": [(0, 9), (1, 64), (0, 0), (1, 65)], "empty row": [(2, 1), (1, 0), (2, 2)],
       "long": [(1, 20000), (1, 7)]}
ROWS = {"prompt": [(33, 33)], "chunk": [(17, 300)], "ragged": [(64, 64), (1, 900), (130, 131), (0, 5), (45, 1000)],
        "empty rows": [(50, 20), (40, 0), (0, 0), (17, 17)], "long": [(20, 5000)], "large": [(300, 1500), (257, 257)]}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens", list(FEW))
def test_attention_of_few_rows(lens, dtype):
    check_attention(R.Case(FEW[lens], heads=8, kv_heads=2, dtype=dtype, seed=1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens", list(ROWS))
def test_attention_of_many_rows(lens, dtype):
    check_attention(R.Case(ROWS[lens], heads=8, kv_heads=2, dtype=dtype, seed=2))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (5, 1), (14, 2), (16, 1), (32, 1), (64, 8), (40, 5)])
@pytest.mark.parametrize("lens", [[(1, 300), (1, 45)], [(37, 190), (2, 9)]])
def test_attention_head_counts(heads, kv_heads, lens):
    check_attention(R.Case(lens, heads=heads, kv_heads=kv_heads, seed=3))


@pytest.mark.parametrize("head_dim", [8, 40, 64, 72, 80, 96, 112, 128, 136, 192, 256])
@pytest.mark.parametrize("lens", [[(1, 300), (1, 45)], [(70, 190), (2, 9)], [(1, 2500)]])
def test_attention_head_sizes(head_dim, lens):
    check_attention(R.Case(lens, heads=4, kv_heads=2, head_dim=head_dim, dtype="f16" if head_dim % 16 else "bf16", seed=4))


@pytest.mark.parametrize("block", [1, 5, 8, 16, 32, 48, 128])
@pytest.mark.parametrize("lens", [[(1, 300), (1, 45)], [(37, 190), (2, 9)]])
def test_attention_block_sizes(block, lens):
    check_attention(R.Case(lens, block=block, seed=5))


@pytest.mark.parametrize("window", [1, 7, 64, 65, 1000, 0xFFFFFFFF])
@pytest.mark.parametrize("lens", [[(1, 1300), (2, 45)], [(150, 700), (2, 9), (40, 20), (300, 300)]])
def test_attention_window(window, lens):
    check_attention(R.Case(lens, head_dim=128, seed=6), window=window, with_sinks=window == 64)


@pytest.mark.parametrize("lens,window", [([(1, 17000)], 16400), ([(2, 5100)], 4000), ([(100, 3300)], 2500), ([(1, 300)], 200)])
def test_attention_window_needs_no_more_workspace(lens, window):
    """Lengths at which the keys without the window would be cut into fewer parts than those within it."""
    check_attention(R.Case(lens, heads=16, kv_heads=8, seed=15), window=window)


@pytest.mark.parametrize("lens", [FEW["ragged"], FEW["empty row"], ROWS["empty rows"], ROWS["ragged"], [(1, 9000)]])
def test_attention_sinks(lens):
    check_attention(R.Case(lens, heads=16, kv_heads=2, seed=7), with_sinks=True)


@pytest.mark.parametrize("lens", [[(1, 300), (1, 40)], [(40, 300), (20, 40)]])
def test_attention_absent_slots(lens):
    """Absent blocks at the start, inside and at the end, one sequence's all: its rows are empty."""
    check_attention(R.Case(lens, absent=[(0, 0), (0, 7), (0, 8), (0, 18), (1, 0), (1, 1), (1, 2)], seed=8))


@pytest.mark.parametrize("n_seq", [1, 150, 700])
def test_attention_batch_sizes(n_seq):
    """Enough sequences that the keys are not split, and a mixed batch."""
    rng = np.random.default_rng(9)
    check_attention(R.Case([(1, int(k)) for k in rng.integers(1, 200, n_seq)], heads=16, kv_heads=8, seed=9))
    check_attention(R.Case([(int(q), int(q + k)) for q, k in zip(rng.integers(0, 9, n_seq), rng.integers(0, 90, n_seq))],
                           heads=16, kv_heads=8, seed=10))


def test_attention_large_logits():
    """Logits in the hundreds, rising along the keys so that the maximum moves in every tile."""
    for lens in ([(1, 1000)], [(60, 1000)]):
        c = R.Case(lens, seed=11)
        slot, off = c.places(0, 1000)
        ramp = torch.linspace(0.1, 40.0, 1000, device="cuda")[:, None, None]
        c.k_cache[slot, :, off] = (torch.ones(1000, 2, 64, device="cuda") * ramp).to(torch.bfloat16)
        q = (torch.ones(c.total, c.heads, 64, device="cuda") * 2.0).to(torch.bfloat16)
        q[:, 1::2] *= -1.0                            # and falling
        check_attention(c, q=q)


def test_attention_strides_and_larger_maxima():
    """Queries and outputs inside wider rows, maxima above the true ones, no lse."""
    for lens in ([(1, 300), (1, 45)], [(37, 190), (2, 9)]):
        c = R.Case(lens, max_q=min(64, sum(q for q, _ in lens)), max_kv=1000, seed=12)
        wide = c.normal(c.total, c.heads + 5, c.head_dim, std=2.0)
        q = wide[:, 2:2 + c.heads]
        room = torch.full((c.total, c.heads + 3, c.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[:, 1:1 + c.heads]
        run_attention(c, q, 0.125, want_lse=False, out=out)
        want, _, tol, _ = R.attention(c, q, 0.125)
        assert ((out.double() - want).abs() <= tol).all()
        assert (room[:, 0] == 7.0).all() and (room[:, 1 + c.heads:] == 7.0).all()


def test_attention_of_a_large_cache():
    """Slots at the end of buffers of more than 2^32 bytes (2^31 elements)."""
    for lens in ([(1, 500)], [(40, 500)]):
        c = R.Case(lens, heads=8, kv_heads=8, head_dim=128, slots=(1 << 32) // (8 * 16 * 128 * 2) + 100, at_end=True, seed=13)
        assert c.k_cache.numel() * 2 > 1 << 32
        check_attention(c)
        del c
        torch.cuda.empty_cache()


def test_attention_repeats_bit_for_bit():
    for lens in ([(1, 5000), (1, 77)], [(40, 5000), (200, 300)]):
        c = R.Case(lens, seed=14)
        q = c.normal(c.total, c.heads, c.head_dim)
        a, la = run_attention(c, q, 0.125)
        for _ in range(3):
            b, lb = run_attention(c, q, 0.125)
            assert torch.equal(a, b) and torch.equal(la, lb)


def test_attention_without_work():
    c = R.Case([(0, 5), (0, 0)])
    K.attention(c.shape, c.batch, 0, 0, 0, 0, 1.0, 0, 0)      # no new token: nothing is looked at
    c = R.Case([])
    assert K.attention_workspace(c.shape, c.batch) == 0
    K.attention(c.shape, c.batch, 0, 0, 0, 0, 1.0, 0, 0)


# ---- attention mass

def run_mass(c, q, scale, lse, last=0, window=0, score_in=None, score_out=None):
    stride = c.max_kv + 3
    if score_out is None:
        score_out = torch.full((len(c.lens), c.kv_heads, stride), 7.0, dtype=torch.float32, device="cuda")
    K.attention_mass(c.shape, c.batch, q.data_ptr(), q.stride(0), c.k_cache.data_ptr(), scale, lse.data_ptr(),
                     score_in.data_ptr() if score_in is not None else 0, score_out.data_ptr(), stride, window=window,
                     last=last, stream=_stream())
    return score_out


@pytest.mark.parametrize("case,kw", [
    (dict(lens=[(1, 1)]), {}), (dict(lens=[(1, 700), (1, 33)], dtype="f16"), {}),
    (dict(lens=[(0, 9), (1, 64), (0, 0), (1, 65)]), {}), (dict(lens=[(50, 20), (40, 0), (17, 17)]), {}),
    (dict(lens=[(64, 64), (1, 900), (130, 131), (0, 5), (45, 1000)]), {}),
    (dict(lens=[(64, 64), (1, 900), (130, 131), (45, 1000)]), dict(last=32)),
    (dict(lens=[(300, 1500), (257, 257)]), dict(window=65)), (dict(lens=[(150, 700), (9, 9)]), dict(window=1, last=7)),
    (dict(lens=[(37, 190)], heads=15, kv_heads=5, head_dim=80, block=5, dtype="f16"), {}),
    (dict(lens=[(37, 190)], heads=7, kv_heads=1, head_dim=256, block=32), dict(last=0xFFFFFFFF, window=0xFFFFFFFF)),
    (dict(lens=[(40, 300), (20, 40)], absent=[(0, 0), (0, 7), (0, 18), (1, 0), (1, 1), (1, 2)]), {}),
    (dict(lens=[(1, 20000)], heads=64, kv_heads=8), {}), (dict(lens=[(2, 3000), (1, 5)]), dict(window=100, last=1)),
    (dict(lens=[(90, 3000), (40, 700)]), dict(window=100, last=3)), (dict(lens=[(2, 900), (0, 70)]), dict(window=33))])
def test_mass(case, kw):
    c = R.Case(seed=20, **case)
    q = c.normal(c.total, c.heads, c.head_dim, std=2.0)
    scale = c.head_dim ** -0.5
    _, lse = run_attention(c, q, scale, window=kw.get("window", 0))
    want, tol = R.mass(c, q, scale, lse, **kw)
    got = run_mass(c, q, scale, lse, **kw)
    start = torch.rand(got.shape, generator=c.g, device="cuda")
    added = run_mass(c, q, scale, lse, score_in=start, **kw)
    again = start.clone()
    run_mass(c, q, scale, lse, score_in=again, score_out=again, **kw)
    for s, (_, kv) in enumerate(c.lens):
        assert ((got[s, :, :kv].double() - want[s, :, :kv]).abs() <= tol[s, :, :kv]).all()
        total = want[s, :, :kv] + start[s, :, :kv].double()
        assert ((added[s, :, :kv].double() - total).abs() <= tol[s, :, :kv] + 2.0 ** -23 * total).all()
        assert torch.equal(again[s, :, :kv], added[s, :, :kv])
        assert (got[s, :, kv:] == 7.0).all() and torch.equal(again[s, :, kv:], start[s, :, kv:])


def test_mass_adds_up():
    """Without sinks every query's weights are 1 together."""
    c = R.Case([(100, 400), (1, 77)], seed=21)
    q = c.normal(c.total, c.heads, c.head_dim, std=2.0)
    _, lse = run_attention(c, q, 0.125)
    got = run_mass(c, q, 0.125, lse)
    group = c.heads // c.kv_heads
    for s, (new, kv) in enumerate(c.lens):
        assert (got[s, :, :kv].double().sum(1) / (new * group) - 1).abs().max().item() < 2.0 ** -16


# ---- eviction

def run_evict(c, keep, score, protect=None, pos=None, in_place=False, score_out=None, pos_out=None):
    def dev(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    keep_dev, protect_dev = dev(keep), dev(protect) if protect is not None else None
    if in_place:
        score_out, pos_out, len_out = score, pos, c.kv_len
    else:
        score_out = torch.full_like(score, 7.0)
        pos_out = torch.full(score.shape, 7, dtype=torch.int32, device="cuda")
        len_out = torch.full_like(c.kv_len, 7)
    w, n = c.workspace(K.evict_workspace)
    K.evict(c.shape, c.batch, keep_dev.data_ptr(), score.data_ptr(), score_out.data_ptr(), score.shape[2],
            c.k_cache.data_ptr(), c.v_cache.data_ptr(), len_out.data_ptr(), w.data_ptr(), n,
            protect=protect_dev.data_ptr() if protect is not None else 0, pos_in=pos.data_ptr() if pos is not None else 0,
            pos_out=pos_out.data_ptr() if pos_out is not None else 0, pos_stride=score.shape[2], stream=_stream())
    return score_out, pos_out, len_out


def check_evict(c, keep, score, protect=None, pos=None, in_place=False):
    k0, v0 = c.k_cache.clone(), c.v_cache.clone()
    s_np = score.cpu().numpy().copy()
    p_np = pos.cpu().numpy().copy() if pos is not None else None
    src, left = R.evict(c, keep, protect, s_np, p_np)
    score_out, pos_out, len_out = run_evict(c, keep, score, protect, pos, in_place)
    assert len_out.cpu().tolist() == left
    for s, (_, kv) in enumerate(c.lens):
        n = left[s]
        slot, off = c.places(s, kv)
        there = c.there(s, kv)
        for h in range(c.kv_heads):
            of = torch.from_numpy(src[s, h]).cuda()
            ok = there[:n] & there[of] if n else there[:0]
            for now, was in ((c.k_cache, k0), (c.v_cache, v0)):
                want = was[slot, h, off].clone()
                want[:n][ok] = was[slot[of], h, off[of]][ok]
                assert torch.equal(now[slot, h, off].view(torch.int16), want.view(torch.int16)), (s, h)
            got = score_out[s, h].cpu().numpy()
            want = s_np[s, h].copy() if in_place else np.full_like(got, 7.0)
            want[:kv] = 0.0 if kv > n else want[:kv]
            want[:n] = s_np[s, h, src[s, h]]
            assert np.array_equal(got.view(np.int32), want.view(np.int32)), (s, h)
            if pos_out is not None:
                p = p_np[s, h] if p_np is not None else np.arange(score.shape[2])
                assert np.array_equal(pos_out[s, h, :n].cpu().numpy(), p[src[s, h]]), (s, h)
    # nothing else was written: the caches differ at places of the batch's kept tokens alone
    changed = (c.k_cache.view(torch.int16) != k0.view(torch.int16)).any(-1)
    for s in range(len(c.lens)):
        if left[s]:
            slot, off = c.places(s, left[s])
            changed[slot, :, off] = False
    assert not changed.any()


def _scores(c, kind, rng):
    shape = (len(c.lens), c.kv_heads, c.max_kv + 3)
    x = rng.standard_normal(shape).astype(np.float32)
    if kind == "ties":
        x = np.floor(np.abs(x) * 2) / 2
    elif kind == "zeros":
        x = np.where(rng.random(shape) < 0.5, 0.0, -0.0).astype(np.float32)
    elif kind == "special":
        x[rng.random(shape) < 0.3] = np.nan
        x[rng.random(shape) < 0.1] = np.inf
        x[rng.random(shape) < 0.1] = -np.inf
        x[rng.random(shape) < 0.1] = np.finfo(np.float32).min
        x[rng.random(shape) < 0.05] = np.float32(1e-45)
        x.view(np.uint32)[rng.random(shape) < 0.05] = 0xFFFFFFFF      # a NaN with its sign set
    elif kind == "rising":
        x = np.broadcast_to(np.arange(shape[2], dtype=np.float32), shape).copy()
    return torch.from_numpy(x).cuda()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["normal", "ties", "zeros", "special", "rising"])
def test_evict(kind, in_place):
    rng = np.random.default_rng(30)
    lens = [(0, 1), (0, 0), (1, 64), (0, 65), (3, 1000), (0, 1025), (0, 5000), (0, 30), (0, 17)]
    keep = [0, 4, 63, 1, 500, 1024, 333, 30, 99]
    c = R.Case(lens, seed=30)
    check_evict(c, keep, _scores(c, kind, rng), in_place=in_place)
    c = R.Case(lens, seed=31, block=5, head_dim=40, kv_heads=3, heads=3, dtype="f16")
    pos = torch.from_numpy(rng.permutation(10 ** 6)[:9 * 3 * 5003].reshape(9, 3, 5003).astype(np.int32)).cuda()
    protect = [0, 0, 900000, 10 ** 6, 500000, 0, 100000, 0, 3]
    check_evict(c, keep, _scores(c, kind, rng), protect=protect, pos=pos, in_place=in_place)


@pytest.mark.parametrize("keep", [-3, 0, 1, 63, 64, 4095, 4096, 20000, 39999, 40000])
def test_evict_amounts(keep):
    rng = np.random.default_rng(32)
    c = R.Case([(0, 40000)], kv_heads=2, head_dim=8, seed=32)
    check_evict(c, [keep], _scores(c, "ties", rng), protect=[39990])


def test_evict_absent_slots():
    rng = np.random.default_rng(33)
    c = R.Case([(0, 300), (0, 40)], absent=[(0, 0), (0, 7), (0, 18), (1, 0), (1, 1), (1, 2)], seed=33)
    check_evict(c, [100, 20], _scores(c, "normal", rng))


def test_evict_again_and_again():
    """Eviction after eviction, in place: positions say which tokens are left, and recent ones stay protected."""
    rng = np.random.default_rng(34)
    c = R.Case([(0, 600)], kv_heads=2, heads=2, seed=34)
    score = _scores(c, "normal", rng)
    pos = torch.arange(603, dtype=torch.int32, device="cuda").repeat(1, 2, 1)
    slot, off = c.places(0, 600)
    first = {h: c.k_cache[slot, h, off].clone() for h in range(2)}
    by_pos = {h: score[0, h].cpu().numpy().copy() for h in range(2)}
    for n in (500, 499, 256, 20):
        run_evict(c, [n], score, protect=[590], pos=pos, in_place=True)
        assert c.kv_len.item() == n
        for h in range(2):
            p = pos[0, h, :n].cpu().numpy()
            want = np.concatenate([np.argsort(-by_pos[h][:590], kind="stable")[:n - 10], np.arange(590, 600)])
            assert set(p.tolist()) == set(want.tolist())
            assert torch.equal(c.k_cache[slot[:n], h, off[:n]], first[h][torch.from_numpy(p).cuda().long()])
            assert np.array_equal(score[0, h, :n].cpu().numpy(), by_pos[h][p])
        c.lens = [(0, n)]


# ---- rotary append

def _angles(n, rot, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.rand(n, max(rot // 2, 1), generator=g, device="cuda", dtype=torch.float64) * 6.28
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _turned(x, angles, positions, rot, interleaved):
    x = x.double().clone()
    first = list(range(0, rot, 2)) if interleaved else list(range(rot // 2))
    second = [i + 1 for i in first] if interleaved else [i + rot // 2 for i in first]
    size = x.abs()
    if rot:
        known = ((positions >= 0) & (positions < len(angles)))[:, None, None]
        c, s = angles[positions.clamp(0, len(angles) - 1).long()].double().unbind(-1)
        c, s = c[:, None], s[:, None]
        a, b = x[..., first], x[..., second]
        x[..., first], x[..., second] = a * c - b * s, b * c + a * s
        size[..., first] = size[..., second] = a.abs() + b.abs()
        x = torch.where(known, x, math.nan)
    return x, size


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head_dim,rot", [(64, 64), (128, 128), (128, 64), (80, 40), (112, 56), (64, 48), (96, 2), (72, 0),
                                          (8, 6), (256, 250), (40, 36)])
def test_rope_append(head_dim, rot, interleaved):
    for dtype, block, heads, kv_heads in (("bf16", 16, 8, 2), ("f16", 5, 3, 3)):
        lens = [(3, 20), (0, 4), (1, 1), (70, 70), (2, 1), (0, 0), (17, 900)]
        c = R.Case(lens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, block=block, dtype=dtype, seed=40,
                   absent=[(3, 1)])
        fused = c.normal(c.total, heads + 2 * kv_heads, head_dim)
        q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
        angles = _angles(50, rot)
        positions = torch.randint(0, 50, (c.total,), generator=c.g, device="cuda", dtype=torch.int32)
        q_out = torch.full((c.total, heads + 1, head_dim), 7.0, dtype=R.DTYPE[dtype], device="cuda")
        pos = torch.full((len(lens), kv_heads, c.max_kv + 2), -5, dtype=torch.int32, device="cuda")
        k0, v0 = c.k_cache.clone(), c.v_cache.clone()
        K.rope_append(c.shape, c.batch, angles.data_ptr(), 50, rot, positions.data_ptr(), k.data_ptr(), k.stride(0),
                      v.data_ptr(), v.stride(0), c.k_cache.data_ptr(), c.v_cache.data_ptr(), q=q.data_ptr(),
                      q_stride=q.stride(0), q_out=q_out.data_ptr(), q_out_stride=q_out.stride(0), pos=pos.data_ptr(),
                      pos_stride=pos.shape[2], interleaved=interleaved, stream=_stream())
        eps = R.EPS[dtype]

        def near(got, x):
            want, size = _turned(x, angles, positions, rot, interleaved)
            tiny = 2.0 ** -25 if dtype == "f16" else 0.0
            assert ((got.double() - want).abs() <= eps * want.abs() * 1.001 + 2.0 ** -22 * size + tiny).all()

        near(q_out[:, :heads], q)
        assert (q_out[:, heads] == 7.0).all()
        got_k, rows = torch.zeros_like(k), torch.zeros(c.total, dtype=torch.bool, device="cuda")
        for s, (new, kv) in enumerate(lens):
            for i in range(new):
                at, t = kv - new + i, int(c.cu_host[s]) + i
                if at < 0:
                    continue
                assert (pos[s, :, at] == positions[t]).all()
                pos[s, :, at] = -5
                if not c.there(s, kv)[at]:
                    continue
                slot, off = int(c.true_table[s, at // block]), at % block
                got_k[t], rows[t] = c.k_cache[slot, :, off], True
                assert torch.equal(c.v_cache[slot, :, off], v[t])
                c.k_cache[slot, :, off], c.v_cache[slot, :, off] = k0[slot, :, off], v0[slot, :, off]
        want, size = _turned(k, angles, positions, rot, interleaved)
        tiny = 2.0 ** -25 if dtype == "f16" else 0.0
        assert ((got_k.double() - want).abs() <= eps * want.abs() * 1.001 + 2.0 ** -22 * size + tiny)[rows].all()
        # and nothing else was written
        assert (pos == -5).all()
        assert torch.equal(c.k_cache.view(torch.int16), k0.view(torch.int16))
        assert torch.equal(c.v_cache.view(torch.int16), v0.view(torch.int16))


def test_rope_append_unknown_position_and_no_query():
    c = R.Case([(4, 10)], heads=4, kv_heads=2, seed=41)
    k, v = c.normal(4, 2, 64), c.normal(4, 2, 64)
    angles = _angles(8, 64)
    positions = torch.tensor([3, -1, 8, 7], dtype=torch.int32, device="cuda")
    K.rope_append(c.shape, c.batch, angles.data_ptr(), 8, 64, positions.data_ptr(), k.data_ptr(), k.stride(0), v.data_ptr(),
                  v.stride(0), c.k_cache.data_ptr(), c.v_cache.data_ptr(), stream=_stream())
    slot, off = c.places(0, 10)
    got = c.k_cache[slot, :, off][6:]
    assert torch.isnan(got[1:3]).all() and torch.isfinite(got[[0, 3]]).all()
    assert torch.equal(c.v_cache[slot, :, off][6:], v)


SCALINGS = [dict(), dict(kind="linear", factor=4.0),
            dict(kind="by_parts", factor=8.0, original_length=8192.0, alpha=1.0, beta=4.0),
            dict(kind="by_parts_index", factor=32.0, original_length=4096.0, alpha=1.0, beta=32.0, magnitude=1.3465735902799727)]


@pytest.mark.parametrize("scaling", SCALINGS, ids=[s.get("kind", "plain") for s in SCALINGS])
@pytest.mark.parametrize("rot", [2, 64, 128, 250])
def test_rope_table(scaling, rot):
    n, base = 131072 if rot == 128 else 3001, 500000.0
    table = torch.empty(n, rot // 2, 2, dtype=torch.float32, device="cuda")
    K.rope_table(table.data_ptr(), n, rot, base=base, stream=_stream(), **scaling)
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    kind, s = scaling.get("kind", "plain"), scaling.get("factor", 1.0)
    turns = scaling.get("original_length", 1.0) * f / (2 * math.pi)
    if kind == "plain":
        g = np.ones_like(f)
    elif kind == "linear":
        g = np.zeros_like(f)
    elif kind == "by_parts":
        g = np.clip((turns - scaling["alpha"]) / (scaling["beta"] - scaling["alpha"]), 0, 1)
    else:
        at = {x: rot / 2 * math.log(scaling["original_length"] / (2 * math.pi * x)) / math.log(base)
              for x in (scaling["alpha"], scaling["beta"])}
        g = np.clip((at[scaling["alpha"]] - np.arange(rot // 2)) / (at[scaling["alpha"]] - at[scaling["beta"]]), 0, 1)
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * torch.from_numpy(f * (g + (1 - g) / s)).cuda()
    want = torch.stack([angle.cos(), angle.sin()], -1) * scaling.get("magnitude", 1.0)
    # rounding to 32 bits, and 2^-52 relative in angles of up to 2^17
    assert (table.double() - want).abs().max().item() <= 1.35 * 2.0 ** -24 + 2.0 ** -33


# ---- together

def test_chain_in_a_graph_and_on_another_stream():
    """Append, attention, mass and eviction captured once and replayed against the eager calls."""
    lens = [(1, 700), (1, 40), (1, 333)]

    def make():
        c = R.Case(lens, heads=8, kv_heads=2, seed=50)
        c.qkv = c.normal(3, 12, 64)
        c.angles, c.positions = _angles(1000, 64), torch.tensor([699, 39, 332], dtype=torch.int32, device="cuda")
        c.q_out, c.out = torch.zeros(3, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 8, 64, dtype=torch.bfloat16, device="cuda")
        c.lse = torch.zeros(8, 3, device="cuda")
        c.score = torch.zeros(3, 2, c.max_kv, device="cuda")
        c.score_out, c.pos = torch.zeros_like(c.score), torch.arange(c.max_kv, dtype=torch.int32, device="cuda").repeat(3, 2, 1)
        c.pos_out, c.len_out = torch.zeros_like(c.pos), torch.zeros_like(c.kv_len)
        c.keep, c.protect = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([300, 300, 300], [690, 30, 320]))
        c.w1, c.n1 = c.workspace(K.attention_workspace)
        c.w2, c.n2 = c.workspace(K.evict_workspace)
        return c

    def step(c):
        s, p = _stream(), c.qkv.data_ptr()
        kc, vc = c.k_cache.data_ptr(), c.v_cache.data_ptr()
        K.rope_append(c.shape, c.batch, c.angles.data_ptr(), 1000, 64, c.positions.data_ptr(), p + 8 * 128, 768, p + 10 * 128,
                      768, kc, vc, q=p, q_stride=768, q_out=c.q_out.data_ptr(), q_out_stride=512, pos=c.pos.data_ptr(),
                      pos_stride=c.max_kv, stream=s)
        K.attention(c.shape, c.batch, c.q_out.data_ptr(), 512, kc, vc, 0.125, c.out.data_ptr(), 512, lse=c.lse.data_ptr(),
                    workspace=c.w1.data_ptr(), workspace_bytes=c.n1, stream=s)
        K.attention_mass(c.shape, c.batch, c.q_out.data_ptr(), 512, kc, 0.125, c.lse.data_ptr(), 0, c.score.data_ptr(),
                         c.max_kv, stream=s)
        K.evict(c.shape, c.batch, c.keep.data_ptr(), c.score.data_ptr(), c.score_out.data_ptr(), c.max_kv, kc, vc,
                c.len_out.data_ptr(), c.w2.data_ptr(), c.n2, protect=c.protect.data_ptr(), pos_in=c.pos.data_ptr(),
                pos_out=c.pos_out.data_ptr(), pos_stride=c.max_kv, stream=s)
        return [x.clone() for x in (c.out, c.lse, c.score, c.score_out, c.pos_out, c.len_out, c.k_cache.view(torch.int16),
                                    c.v_cache.view(torch.int16))]

    eager, graphed = make(), make()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        streamed = step(make())
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(graphed)
    for i in range(3):
        x = torch.randn(3, 12, 64, device="cuda").to(torch.bfloat16) if i else eager.qkv.clone()
        eager.qkv.copy_(x)
        graphed.qkv.copy_(x)
        want = step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
        if i == 0:
            for a, b in zip(streamed, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("lens,heads,head_dim", [([(3, 200), (2, 9)], 8, 64), ([(4, 500)], 8, 128), ([(100, 333), (70, 70)], 8, 64),
                                                 ([(300, 300)], 2, 128), ([(40, 90)], 4, 256), ([(3, 90)], 4, 200)])
def test_attention_unseen_values_do_not_leak(lens, heads, head_dim, window, dtype):
    """Infinities and NaN among keys and values of tokens that some queries see and others, in the same tile, do not:
    the others are as without them, and those that see a value's element are not finite there."""
    c = R.Case(lens, heads=heads, kv_heads=2, head_dim=head_dim, dtype=dtype, seed=60)
    q = c.normal(c.total, heads, head_dim, std=2.0)
    want, want_lse, tol, tol_lse = R.attention(c, q, 0.1, window)
    marks = {}
    for s, (new, kv) in enumerate(lens):
        slot, off = c.places(s, kv)
        for at, value in ((kv - 1, math.nan), (kv - 2, math.inf), (max(0, kv - new - 30), -math.inf), (kv - new, math.inf)):
            marks.setdefault(s, []).append(at)
            c.v_cache[slot[at], 1, off[at], 5] = value
            c.v_cache[slot[at], 1, off[at], head_dim - 1] = value
        c.k_cache[slot[kv - 1], 0, off[kv - 1], 3] = math.nan         # a key of the first KV head
    out, lse = run_attention(c, q, 0.1, window)
    group = heads // 2
    for s, (new, kv) in enumerate(lens):
        for i in range(new):
            t, index = int(c.cu_host[s]) + i, kv - new + i
            sees = [index >= at and (not window or at > index - window) for at in marks[s]]
            ok = torch.ones(heads, head_dim, dtype=torch.bool, device="cuda")
            if any(sees):
                ok[group:, 5] = ok[group:, head_dim - 1] = False
            if i == new - 1:
                ok[:group] = False
                assert torch.isnan(out[t, :group]).all() and torch.isnan(lse[:group, t]).all()
            off = (out[t].double() - want[t]).abs()
            assert (off <= tol[t])[ok].all(), (s, i)
            assert not torch.isfinite(out[t])[group:][~ok[group:]].any()
            heads_ok = slice(group if i == new - 1 else 0, heads)
            assert ((lse[heads_ok, t].double() - want_lse[heads_ok, t]).abs() <= tol_lse[heads_ok, t]).all()
