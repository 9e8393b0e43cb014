"""The operators on pages of either kind and on drafted tokens against plain forms in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_ops_ref as R   # noqa: E402
import pages_ref as P   # noqa: E402
from paper_2606_14779_amd import kvpool as K   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- attention

def _attend(c, q, scale, tree=None, window=0, sinks=None, out=None, lse=None, work=None):
    out = torch.full((c.total, c.heads, c.head_dim), 7.0, dtype=R.DTYPE[c.dtype], device="cuda") if out is None else out
    lse = torch.full((c.heads, c.total), 7.0, dtype=torch.float32, device="cuda") if lse is None else lse
    w, n = c.workspace(K.attention_pages_workspace) if work is None else (work, work.numel())
    K.attention_pages(c.shape, c.batch, c.pages, q.data_ptr(), q.stride(0), scale, out.data_ptr(), out.stride(0),
                      tree=tree.data_ptr() if tree is not None else 0, tree_words=tree.shape[1] if tree is not None else 0,
                      window=window, sinks=sinks.data_ptr() if sinks is not None else 0, lse=lse.data_ptr(),
                      workspace=w.data_ptr(), workspace_bytes=n, stream=_stream())
    return out, lse


def _check(got, want):
    out, lse = got
    o, e, tol, tol_e = want
    empty = e == -math.inf
    assert (lse[empty] == -math.inf).all() and (out.float().permute(1, 0, 2)[empty] == 0).all()
    assert ((lse.double() - e).abs()[~empty] <= tol_e[~empty]).all()
    bad = (out.double() - o).abs() > tol
    assert not bad.any(), (out.double() - o).abs().max().item()


LENS = {                                             # (new, cached): rows for every kernel, lengths of 0 and 1
    "few": [(1, 1), (2, 300), (0, 17), (1, 129), (2, 2), (2, 63)],
    "few, long": [(1, 5000), (2, 33)],
    "tile of 64": [(9, 9), (16, 700), (1, 40), (0, 0), (3, 64)],
    "tile of 64, long": [(12, 9000)],
    "tile of 128": [(30, 31), (20, 333), (1, 1)],
    "tile of 256": [(33, 500), (70, 70), (1, 64), (64, 129), (0, 3)],
    "tile of 256, long": [(130, 7000), (65, 200)],
}
SHAPES = [(8, 2, 64, 16), (4, 1, 128, 16), (6, 2, 80, 8), (4, 1, 256, 16), (8, 2, 24, 5), (4, 4, 136, 1)]


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", list(LENS))
def test_attention(kind, tree, shape, lens):
    h, hk, d, block = shape
    for dtype, window, sinks in (("bf16", 0, False), ("f16", 50, True)):
        c = P.Case(LENS[lens], kind, heads=h, kv_heads=hk, head_dim=d, block=block, dtype=dtype, seed=len(lens) + d)
        q = c.normal(c.total, h, d, std=2.0)
        sink = c.normal(h, std=2.0, to=torch.float32) if sinks else None
        bits, mask = c.tree(3) if tree else (None, None)
        scale = d ** -0.5
        got = _attend(c, q, scale, bits, window, sink)
        _check(got, P.attention(c, q, scale, window, sink, mask))
        again = _attend(c, q, scale, bits, window, sink)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("group", [1, 3, 5, 16, 33])
def test_attention_groups_strides_and_absent_blocks(kind, group):
    lens = [(5, 200), (17, 90), (1, 333), (66, 66)]
    c = P.Case(lens, kind, heads=2 * group, kv_heads=2, head_dim=64, block=16, seed=group, absent=[(0, 3), (1, 5), (2, 0), (3, 1)])
    q = c.normal(c.total, 2 * group + 3, 80, std=2.0)[:, :2 * group].contiguous()   # heads of 64 in a wider row
    wide = torch.full((c.total, 2 * group * 64 + 24), math.nan, dtype=R.DTYPE[c.dtype], device="cuda")
    q = wide[:, 8:8 + 2 * group * 64].view(c.total, 2 * group, 64).copy_(q[..., :64])
    out = torch.full((c.total, 2 * group * 64 + 16), 5.0, dtype=R.DTYPE[c.dtype], device="cuda")
    to = out[:, :2 * group * 64].view(c.total, 2 * group, 64)
    for tree in (False, True):
        bits, mask = c.tree(5, words=3) if tree else (None, None)
        _check(_attend(c, q, 0.125, bits, out=to), P.attention(c, q, 0.125, mask=mask))
        assert (out[:, 2 * group * 64:] == 5.0).all()


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("lens", [[(4, 100), (3, 3)], [(40, 300), (12, 12)], [(90, 400), (7, 700)]], ids=str)
def test_a_causal_tree_is_no_tree(kind, lens):
    """A mask of the tokens up to each one's own is the causal one, under a window too: their depths are their places."""
    c = P.Case(lens, kind, seed=9)
    q = c.normal(c.total, 8, 64, std=2.0)
    words = -(-c.max_q // 64)
    mask = np.zeros((c.total, words * 64), bool)
    for s, (new, _) in enumerate(lens):
        mask[c.cu_host[s]:c.cu_host[s + 1], :new] = np.tril(np.ones((new, new), bool))
    bits = torch.from_numpy(np.packbits(mask, axis=1, bitorder="little").view(np.int64).copy()).cuda()
    mask = torch.from_numpy(mask).cuda()
    for window in (0, 100):
        want = P.attention(c, q, 0.125, window)
        _check(_attend(c, q, 0.125, None, window), want)
        _check(_attend(c, q, 0.125, bits, window), P.attention(c, q, 0.125, window, mask=mask))
        if not window:
            _check(_attend(c, q, 0.125, bits), want)


def test_pages_of_16_bits_without_a_tree_are_those_of_attention():
    c = P.Case([(1, 700), (40, 400), (3, 3)], "16", seed=4)
    q = c.normal(c.total, 8, 64, std=2.0)
    out, lse = _attend(c, q, 0.125, window=60)
    other, other_lse = torch.empty_like(out), torch.empty_like(lse)
    w, n = c.workspace(K.attention_workspace)
    K.attention(c.shape, c.batch, q.data_ptr(), q.stride(0), c.buffers[0].raw.data_ptr(), c.buffers[1].raw.data_ptr(), 0.125,
                other.data_ptr(), other.stride(0), window=60, lse=other_lse.data_ptr(), workspace=w.data_ptr(),
                workspace_bytes=n, stream=_stream())
    assert torch.equal(out, other) and torch.equal(lse, other_lse)


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("lens", [[(4, 100), (3, 37)], [(15, 300), (9, 40)], [(70, 400), (30, 90)]], ids=str)
def test_values_that_only_some_rows_see(kind, value, lens):
    """An infinity or NaN among the new tokens' values and keys: rows that do not see the token are as if it were not
    there, those that do show it.

    As if it were not there, but for the point that their weights refer to, which moves when that of another row of the
    wave does: both are within the plain form's tolerance, and without an infinite logit the bits are the same."""
    c = P.Case(lens, kind, seed=11)
    q = c.normal(c.total, 8, 64, std=1.0)
    bits, mask = c.tree(6)
    clean = _attend(c, q, 0.125, bits)
    o, e, tol, tol_e = P.attention(c, q, 0.125, mask=mask)
    for cache in (1, 0):                             # values, then keys
        b = c.buffers[cache]
        keep = b.raw.clone()
        hit = torch.zeros(c.total, dtype=torch.bool, device="cuda")
        for s, (new, kv) in enumerate(lens):
            j = new // 2
            slot, off = c.places(s, kv)
            x = b.rows(slot[kv - new + j:kv - new + j + 1], off[kv - new + j:kv - new + j + 1])
            x[..., 5] = value
            b.put(slot[kv - new + j:kv - new + j + 1], off[kv - new + j:kv - new + j + 1], x)
            hit[int(c.cu_host[s]):int(c.cu_host[s + 1])] = mask[int(c.cu_host[s]):int(c.cu_host[s + 1]), j]
        out, lse = _attend(c, q, 0.125, bits)
        assert hit.any() and not hit.all()
        assert ((out.double() - o).abs() <= tol)[~hit].all() and ((lse.double() - e).abs() <= tol_e)[:, ~hit].all()
        if cache == 1 or math.isnan(value):
            assert torch.equal(out[~hit], clean[0][~hit]) and torch.equal(lse[:, ~hit], clean[1][:, ~hit])
        if cache == 1:
            assert torch.equal(lse, clean[1])        # values do not enter it
            shown = out[hit][..., 5]
            assert (torch.isnan(shown) if kind == "e4m3" or math.isnan(value) else torch.isinf(shown)).all()
            others = torch.cat([out[hit][..., :5], out[hit][..., 6:]], -1)
            assert torch.isfinite(others).all()
        b.raw.copy_(keep)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_reads_every_byte_as_it_stands(dtype):
    """One key and value: the output is the value, exactly, for every finite element and a range of exponents."""
    c = P.Case([(1, 1)] * 8, heads=2, kv_heads=2, head_dim=256, block=1, dtype=dtype, spare=0)
    elements, scales = c.buffers[1].elements().view(torch.uint8), c.buffers[1].scales()
    byte = torch.arange(256, device="cuda").to(torch.uint8)
    byte[(byte & 0x7F) == 0x7F] = 0
    least, most = P.LIMITS[dtype]
    want = []
    for i in range(8):
        slot = int(c.true_table[i, 0])
        elements[slot] = byte
        e = torch.tensor([least + (most - 1 - least) * (i * 8 + b) // 63 for b in range(8)], device="cuda")   # most: finite to 240
        scales[slot] = (e + 127).to(torch.uint8)
        want.append(P.unpack(elements[slot].view(torch.float8_e4m3fn), scales[slot])[:, 0])
    q = c.normal(8, 2, 256)
    c.buffers[0].raw.zero_()
    out, _ = _attend(c, q, 1.0)
    assert torch.equal(out.double(), torch.stack(want))


@pytest.mark.parametrize("new", [1, 20])
def test_caches_of_more_than_2_32_bytes(new):
    """Slots past 2^32 bytes of 8-bit pages; only the last ones hold tokens."""
    slots = (1 << 32) // (2 * 16 * 68) + 100
    c = P.Case([(new, 600), (1, 70)], heads=8, kv_heads=2, seed=2, slots=slots, at_end=True)
    q = c.normal(c.total, 8, 64)
    bits, mask = c.tree(2)
    _check(_attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))


@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_many_sequences(kind):
    rng = np.random.default_rng(0)
    for n, most in ((700, 2), (130, 30)):
        lens = [(int(q), int(q + rng.integers(0, 90))) for q in rng.integers(0, most, n)]
        c = P.Case(lens, kind, heads=8, kv_heads=2, head_dim=64, seed=n)
        q = c.normal(c.total, 8, 64, std=2.0)
        bits, mask = c.tree(n)
        _check(_attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))


def test_a_large_tree():
    c = P.Case([(1000, 1500), (129, 129)], heads=2, kv_heads=1, head_dim=64, seed=1)
    q = c.normal(c.total, 2, 64, std=2.0)
    bits, mask = c.tree(1)
    for window in (0, 200):
        _check(_attend(c, q, 0.125, bits, window), P.attention(c, q, 0.125, window, mask=mask))


def test_rows_that_see_nothing():
    """No token before the new ones, and masks that show nothing of them: 0 and -inf, or the sink's."""
    c = P.Case([(3, 3), (40, 40), (2, 9)], seed=3)
    q = c.normal(c.total, 8, 64)
    bits = torch.zeros(c.total, 1, dtype=torch.int64, device="cuda")
    mask = torch.zeros(c.total, 64, dtype=torch.bool, device="cuda")
    _check(_attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))
    sinks = c.normal(8, to=torch.float32)
    out, lse = _attend(c, q, 0.125, bits, sinks=sinks)
    _check((out, lse), P.attention(c, q, 0.125, sinks=sinks, mask=mask))
    assert torch.allclose(lse[:, :43], sinks[:, None].expand(-1, 43), rtol=1e-6, atol=0)


@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_captured_on_another_stream(kind):
    """A graph of append, attention and commit, replayed several times among eager work, against the same calls eager."""
    c = P.Case([(6, 400), (20, 300)], kind, seed=8)
    q, k, v = (c.normal(c.total, n, 64) for n in (8, 2, 2))
    table = torch.empty(1000, 32, 2, dtype=torch.float32, device="cuda")
    K.rope_table(table.data_ptr(), 1000, 64, stream=_stream())
    bits, _ = c.tree(4)
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(8, c.total, dtype=torch.float32, device="cuda")
    positions = torch.arange(c.total, dtype=torch.int32, device="cuda")
    path = _dev([0, 2, 3] + [0] * 3 + [1, 4, 5, 9, 19] + [0] * 15)
    accepted, left = _dev([3, 5]), _dev([0, 0])
    work, _ = c.workspace(K.attention_pages_workspace)
    first = [b.raw.clone() for b in c.buffers]

    def calls():
        K.norm_rope_append(c.shape, c.batch, c.pages, table.data_ptr(), 1000, 64, positions.data_ptr(), k.data_ptr(), 128,
                           v.data_ptr(), 128, norm=K.HeadNorm(0, 0, 1e-6), q=q.data_ptr(), q_stride=512,
                           q_out=q_out.data_ptr(), q_out_stride=512, stream=_stream())
        _attend(c, q_out, 0.125, bits, out=out, lse=lse, work=work)
        K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), left.data_ptr(), stream=_stream())

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q_out, out, lse, left, *(b.raw for b in c.buffers))]
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for _ in range(4):
        for t in (q_out, out, lse):
            t.fill_(3.0)
        for b, f in zip(c.buffers, first):
            b.raw.copy_(f)
        torch.cuda.synchronize()
        graph.replay()
        (torch.ones(1000, device="cuda") * 2).sum()
        torch.cuda.synchronize()
        for a, b in zip((q_out, out, lse, left, *(b.raw for b in c.buffers)), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# ---- append

def _table(n, rot):
    t = torch.empty(n, max(rot // 2, 1), 2, dtype=torch.float32, device="cuda")
    if rot:
        K.rope_table(t.data_ptr(), n, rot, base=10000.0, stream=_stream())
    return t


def _append(c, qkv, table, rot, positions, *, norm=None, axes=None, interleaved=False, q=True, pos=None):
    h, hk, d = c.heads, c.kv_heads, c.head_dim
    q_out = torch.full((c.total, h, d), 3.0, dtype=R.DTYPE[c.dtype], device="cuda")
    at, stride = qkv.data_ptr(), qkv.stride(0)
    K.norm_rope_append(c.shape, c.batch, c.pages, table.data_ptr() if rot else 0, table.shape[0], rot, positions.data_ptr(),
                       at + h * d * 2, stride, at + (h + hk) * d * 2, stride, norm=norm, axes=axes, q=at if q else 0,
                       q_stride=stride, q_out=q_out.data_ptr() if q else 0, q_out_stride=h * d,
                       pos=pos.data_ptr() if pos is not None else 0, pos_stride=c.max_kv, interleaved=interleaved,
                       stream=_stream())
    return q_out


def _near(got, want, err, dtype):
    """Rounded once to 16 bits, after an error of 32-bit arithmetic."""
    eps = R.EPS[dtype]
    least = 2.0 ** -25 if dtype == "f16" else 0.0
    return ((got.double() - want).abs() <= want.abs() * eps + err * (1 + eps) + least).all()


def _near8(b, slot, off, want, err):
    """Elements of 8 bits: half a step of 3 bits of mantissa, or of the least step, after an error of 32-bit arithmetic;
    the exponent is the least that holds the largest, give or take that error."""
    got = b.rows(slot, off)
    e = b.scales()[slot, :, off].int() - 127
    d = want.shape[-1]
    used = -(-d // 32)
    lo, hi = P.exponents(want * (1 - 2.0 ** -18), b.dtype), P.exponents(want * (1 + 2.0 ** -18), b.dtype)
    assert ((e[..., :used] >= lo) & (e[..., :used] <= hi)).all() and (e[..., used:] == -127).all()
    step = P.pow2(e[..., :used] - 10).repeat_interleave(32, -1)[..., :d]
    top = torch.where(e[..., :used] == P.LIMITS[b.dtype][1], 240.0, 448.0).double().repeat_interleave(32, -1)[..., :d] * step * 1024
    w = torch.maximum(torch.minimum(want, top), -top)
    return ((got - w).abs() <= torch.maximum(w.abs() * 2.0 ** -4, step) + err * 1.0625).all()


APPEND = [  # rot, interleaved, axes, norm, weights
    (1.0, False, 1, True, True), (1.0, False, 3, True, True), (1.0, True, 2, True, False), (0.5, False, 4, False, True),
    (0.5, True, 1, True, True), (0.0, False, 1, True, True), (0.0, False, 1, False, True), (-1, False, 3, True, True),
]


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("shape", [(8, 2, 64, 16), (16, 4, 128, 16), (6, 2, 80, 8), (3, 1, 256, 4), (4, 4, 24, 5), (2, 1, 8, 1),
                                   (70, 7, 136, 3)], ids=str)
@pytest.mark.parametrize("how", APPEND, ids=str)
def test_append(kind, shape, how):
    h, hk, d, block = shape
    part, interleaved, n_axes, normed, weights = how
    rot = int(d * part) // 2 * 2 if part >= 0 else d - 6        # d - 6: pairs that lie anyhow
    lens = [(3, 40), (0, 7), (1, 1), (17, 17), (2, 90)]
    for dtype in ("bf16", "f16"):
        c = P.Case(lens, kind, heads=h, kv_heads=hk, head_dim=d, block=block, dtype=dtype, seed=d, absent=[(3, 0)])
        before = [b.raw.clone() for b in c.buffers]
        qkv = c.normal(c.total, h + 2 * hk + 1, d, std=3.0)
        table = _table(200, rot)
        positions = torch.randint(0, 200, (n_axes, c.total), dtype=torch.int32, device="cuda", generator=c.g)
        axis_of = [(j * 7) % n_axes for j in range(128)]
        q_w, k_w = (c.normal(d) if weights else None for _ in range(2))
        norm = K.HeadNorm(*(w.data_ptr() if w is not None else 0 for w in (q_w, k_w)), 1e-5) if normed else None
        pos = torch.full((len(lens), hk, c.max_kv), -5, dtype=torch.int32, device="cuda")
        q_out = _append(c, qkv, table, rot, positions, norm=norm, axes=K.RopeAxes(n_axes, axis_of) if n_axes > 1 else None,
                        interleaved=interleaved, pos=pos)
        args = (1e-5, table, positions, axis_of, rot, interleaved, normed)
        want, err = P.turned(qkv[:, :h], q_w, *args)
        assert _near(q_out, want, err, dtype)
        want, err = P.turned(qkv[:, h:h + hk], k_w, *args)
        value = qkv[:, h + hk:h + 2 * hk]
        want_pos = torch.full_like(pos, -5)
        written = [torch.zeros(b.raw.shape[0], hk, block, dtype=torch.bool, device="cuda") for b in c.buffers]
        for s, (new, kv) in enumerate(lens):
            rows = slice(int(c.cu_host[s]), int(c.cu_host[s + 1]))
            want_pos[s, :, kv - new:kv] = positions[0, rows]
            there = c.there(s, kv)[kv - new:]
            slot, off = (x[kv - new:][there] for x in c.places(s, kv))
            for b, w, r, mark in zip(c.buffers, (want, value.double()), (err, torch.zeros_like(err)), written):
                mark[slot, :, off] = True
                if kind == "16":
                    assert _near(b.elements()[slot, :, off], w[rows][there], r[rows][there], dtype)
                else:
                    assert _near8(b, slot, off, w[rows][there], r[rows][there])
            if len(slot):                            # values are rounded, nothing else
                exact = P.Buffer(kind, c.slots, hk, block, d, dtype)
                exact.put(slot, off, value[rows][there])
                assert torch.equal(c.buffers[1].elements().view(torch.uint8)[slot, :, off],
                                   exact.elements().view(torch.uint8)[slot, :, off])
        assert torch.equal(pos, want_pos)
        for b, was, mark in zip(c.buffers, before, written):   # and nothing else was written
            if kind == "e4m3":
                b.elements().view(torch.uint8)[mark] = 0
                b.scales()[mark] = 0
                other = P.Buffer(kind, c.slots, hk, block, d, dtype)
                other.raw = was
                other.elements().view(torch.uint8)[mark] = 0
                other.scales()[mark] = 0
                assert torch.equal(b.raw, was)
            else:
                b.elements()[mark] = 0
                was.view(R.DTYPE[dtype]).view(b.dims)[mark] = 0
                assert torch.equal(b.raw, was)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (32, False), (44, False), (20, True), (0, False)])
def test_append_without_norm_is_rope_append(dtype, rot, interleaved):
    c = P.Case([(5, 70), (33, 33)], "16", dtype=dtype, seed=rot)
    qkv = c.normal(c.total, 12, 64, std=2.0)
    table, positions = _table(100, rot), torch.arange(c.total, dtype=torch.int32, device="cuda") * 2
    q_out = _append(c, qkv, table, rot, positions, interleaved=interleaved)
    other, k_cache, v_cache = torch.empty_like(q_out), c.buffers[0].raw.clone(), c.buffers[1].raw.clone()
    at, row = qkv.data_ptr(), qkv.stride(0)
    K.rope_append(c.shape, c.batch, table.data_ptr() if rot else 0, 100, rot, positions.data_ptr(), at + 8 * 64 * 2, row,
                  at + 10 * 64 * 2, row, k_cache.data_ptr(), v_cache.data_ptr(), q=at, q_stride=row, q_out=other.data_ptr(),
                  q_out_stride=512, interleaved=interleaved, stream=_stream())
    assert torch.equal(q_out, other)
    assert torch.equal(c.buffers[0].raw, k_cache) and torch.equal(c.buffers[1].raw, v_cache)


@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_append_of_unknown_positions(kind):
    """On any axis: NaN queries and keys; values and the other tokens as they are."""
    c = P.Case([(4, 30)], kind, seed=1)
    qkv, table = c.normal(4, 12, 64), _table(50, 64)
    positions = _dev([[1, 50, 3, 4], [1, 2, -1, 4]])
    axes = K.RopeAxes(2, [0] * 32)                   # the second is no pair's
    q_out = _append(c, qkv, table, 64, positions, axes=axes)
    bad = torch.tensor([False, True, True, False], device="cuda")
    assert torch.isnan(q_out[bad]).all() and torch.isfinite(q_out[~bad]).all()
    slot, off = (x[26:] for x in c.places(0, 30))
    keys, values = (b.rows(slot, off) for b in c.buffers)
    assert torch.isnan(keys[bad]).all() and torch.isfinite(keys[~bad]).all() and torch.isfinite(values).all()
    _append(c, qkv, table, 0, positions, axes=axes, q=False)     # without a rotation too
    assert torch.isnan(c.buffers[0].rows(slot, off)[bad]).all()


@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_norms_at_the_ends_of_the_range(kind):
    """Heads of very large and very small elements, of zeros, and with what is no number."""
    c = P.Case([(8, 8)], kind, heads=1, kv_heads=1, head_dim=128, seed=2)
    x = c.normal(8, 128, to=torch.float32)
    x[0] *= 2.0 ** 120
    x[1] *= 2.0 ** -110
    x[2] = 0.0
    x[3, 7] = math.nan
    x[4, 9] = math.inf
    x[5] = 0.0
    x[5, 100] = 2.0 ** -120
    x[6] = 2.0 ** 64
    qkv = x.to(torch.bfloat16)[:, None].expand(8, 3, 128).contiguous()
    positions, table = torch.zeros(8, dtype=torch.int32, device="cuda"), _table(4, 128)
    for eps in (0.0, 1e-6):
        q_out = _append(c, qkv, table, 128, positions, norm=K.HeadNorm(0, 0, eps))[:, 0]
        want, err = P.turned(qkv[:, :1], None, eps, table, positions[None], [0] * 64, 128, False, True)
        want, err = want[:, 0], err[:, 0]
        keys = c.buffers[0].rows(*c.places(0, 8))[:, 0]
        for i in (0, 1, 5, 6) if eps == 0 else (0, 2, 6):
            assert _near(q_out[i], want[i], err[i] * 2 + 1e-38, "bf16"), i
            if kind == "16":
                assert torch.equal(keys[i], q_out[i].double())
        assert torch.isnan(q_out[2]).all() == (eps == 0)         # 0 / 0
        assert torch.isnan(q_out[3]).all()
        assert torch.isnan(q_out[4, 9]) and (q_out[4, [i for i in range(128) if i not in (9, 73)]] == 0).all()
        values = c.buffers[1].rows(*c.places(0, 8))[:, 0]
        if kind == "e4m3":                           # infinities and NaN are NaN, the others as without them
            assert torch.isnan(values[3, 7]) and torch.isnan(values[4, 9])
            ok = ~torch.isnan(values)
            assert ok.sum() == 8 * 128 - 2
            y, e = P.pack(qkv[:, 2], "bf16")
            assert torch.equal(values[ok], P.unpack(y, e)[ok])
        else:
            assert torch.equal(values.nan_to_num(1.0, 2.0), qkv[:, 2].double().nan_to_num(1.0, 2.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantised_values_of_every_size(dtype):
    """Rows of 32 from the type's smallest to its largest: the exact bits, all finite when read."""
    most = torch.finfo(R.DTYPE[dtype]).max
    least = 2.0 ** -24 if dtype == "f16" else 2.0 ** -126
    rows = int(math.log2(most / least)) + 2
    c = P.Case([(rows, rows)], heads=1, kv_heads=1, head_dim=96, dtype=dtype, seed=5)
    x = torch.rand(rows, 96, device="cuda", generator=c.g, dtype=torch.float64) * 2 - 1
    x[:, 31] = 1.0
    x[:, 40:64] *= 2.0 ** -9
    x = x * torch.minimum(torch.pow(2.0, torch.arange(rows, device="cuda").double()) * least, torch.tensor(most).double())[:, None]
    x[-1, :] = most * torch.sign(x[-1])
    x = x.to(R.DTYPE[dtype])
    qkv = x[:, None].expand(rows, 3, 96).contiguous()
    _append(c, qkv, _table(4, 0), 0, torch.zeros(rows, dtype=torch.int32, device="cuda"), q=False)
    want, e = P.pack(x, dtype)
    slot, off = c.places(0, rows)
    for b in c.buffers:
        assert torch.equal(b.elements().view(torch.uint8)[slot, 0, off], want.view(torch.uint8))
        assert torch.equal(b.scales()[slot, 0, off], e)
        back = b.rows(slot, off)[:, 0]
        assert torch.equal(back.to(R.DTYPE[dtype]).double(), back) and torch.isfinite(back).all()
        step = P.pow2(e[:, :3].int() - 137).repeat_interleave(32, -1)
        assert ((back - x.double()).abs() <= torch.maximum(x.double().abs() * 2.0 ** -4, step)).all()


# ---- conversion

@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("shape", [(2, 64, 16), (8, 128, 16), (3, 80, 8), (1, 256, 4), (2, 24, 5), (5, 8, 1), (1, 136, 130),
                                   (2, 32, 64)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_convert(back, shape, dtype):
    hk, d, block = shape
    lens = [(0, 0), (0, 1), (0, 300), (0, 65), (0, 64)]
    a, b = ("e4m3", "16") if back else ("16", "e4m3")
    c = P.Case(lens, a, heads=hk, kv_heads=hk, head_dim=d, block=block, dtype=dtype, seed=d + back, absent=[(2, 0)])
    blocks = [-(-kv // block) for _, kv in lens]
    slots = sum(blocks) + 2
    order = torch.randperm(slots, generator=torch.Generator().manual_seed(1)).tolist()
    table = np.full((len(lens), c.stride + 3), -1, np.int32)
    for s, n in enumerate(blocks):
        table[s, :n] = [order.pop() for _ in range(n)]
    if blocks[3] > 1:
        table[3, 1] = slots                          # absent where it is to go
    to = [P.Buffer(b, slots, hk, block, d, dtype) for _ in range(2)]
    first = [0, 0, 7, 0, 200]
    table_dev, first_dev = _dev(table.tolist()), _dev(first)
    K.convert_pages(c.shape, c.batch, c.pages, K.Pages(b, *(x.raw.data_ptr() for x in to)), table_dev.data_ptr(),
                    table.shape[1], slots, first=first_dev.data_ptr(), stream=_stream())
    want = [P.Buffer(b, slots, hk, block, d, dtype) for _ in range(2)]
    for s, (_, kv) in enumerate(lens):
        if not kv:
            continue
        slot, off = c.places(s, kv)
        dest = torch.from_numpy(np.repeat(table[s], block)[:kv].astype(np.int64)).cuda()
        moves = c.there(s, kv) & (dest >= 0) & (dest < slots) & (torch.arange(kv, device="cuda") >= first[s])
        for source, out in zip(c.buffers, want):
            if moves.any():
                out.put(dest[moves], off[moves], source.rows(slot[moves], off[moves]))
    for got, w in zip(to, want):
        assert torch.equal(got.raw, w.raw)
    K.convert_pages(c.shape, c.batch, c.pages, K.Pages(b, *(x.raw.data_ptr() for x in to)), table_dev.data_ptr(),
                    table.shape[1], slots, stream=_stream())
    assert torch.equal(to[0].rows(*(torch.tensor([x], device="cuda") for x in (int(table[1, 0]), 0))),
                       want[0].rows(*(torch.tensor([x], device="cuda") for x in (int(table[1, 0]), 0))))


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("before", [False, True])
@pytest.mark.parametrize("shape", [(2, 64, 16), (3, 80, 8), (1, 136, 130)], ids=str)
def test_convert_without_a_first_token(back, before, shape):
    """All cached tokens of all sequences and nothing else, into buffers as they were, or after a call that left out the
    first ones."""
    hk, d, block = shape
    lens = [(0, 90), (0, 1), (0, 300), (0, 0), (0, 64)]
    a, b = ("e4m3", "16") if back else ("16", "e4m3")
    c = P.Case(lens, a, heads=hk, kv_heads=hk, head_dim=d, block=block, seed=d)
    slots = c.slots + 5
    table = np.full((len(lens), c.stride), -1, np.int32)
    order = torch.randperm(slots, generator=torch.Generator().manual_seed(2)).tolist()
    for s, (_, kv) in enumerate(lens):
        n = -(-kv // block)
        table[s, :n] = [order.pop() for _ in range(n)]
    to, want = ([P.Buffer(b, slots, hk, block, d, "bf16") for _ in range(2)] for _ in range(2))
    pages = K.Pages(b, *(x.raw.data_ptr() for x in to))
    table_dev, first = _dev(table.tolist()), _dev([7, 1, 299, 0, 200])
    if before:
        K.convert_pages(c.shape, c.batch, c.pages, pages, table_dev.data_ptr(), table.shape[1], slots, first=first.data_ptr(),
                        stream=_stream())
    K.convert_pages(c.shape, c.batch, c.pages, pages, table_dev.data_ptr(), table.shape[1], slots, stream=_stream())
    for s, (_, kv) in enumerate(lens):
        if kv:
            slot, off = c.places(s, kv)
            dest = torch.from_numpy(np.repeat(table[s], block)[:kv].astype(np.int64)).cuda()
            for source, out in zip(c.buffers, want):
                out.put(dest, off, source.rows(slot, off))
    for got, w in zip(to, want):
        assert torch.equal(got.raw, w.raw)


def test_there_and_back_again():
    """8 bits to 16 and back to 8 gives the same bits: what was written is what is read."""
    for dtype in ("bf16", "f16"):
        c = P.Case([(0, 500)], "e4m3", dtype=dtype, head_dim=128, seed=3)
        wide = [P.Buffer("16", c.slots, 2, 16, 128, dtype) for _ in range(2)]
        thin = [P.Buffer("e4m3", c.slots, 2, 16, 128, dtype) for _ in range(2)]
        p16, p8 = (K.Pages(k, *(x.raw.data_ptr() for x in b)) for k, b in (("16", wide), ("e4m3", thin)))
        args = (c.table_dev.data_ptr(), c.stride, c.slots)
        K.convert_pages(c.shape, c.batch, c.pages, p16, *args, stream=_stream())
        K.convert_pages(c.shape, c.batch, p16, p8, *args, stream=_stream())
        slot, off = c.places(0, 500)
        for a, b in zip(c.buffers, thin):
            assert torch.equal(a.rows(slot, off), b.rows(slot, off))


# ---- commit

@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("shape", [(2, 64, 16), (4, 128, 16), (1, 80, 8), (2, 256, 3), (3, 8, 1), (2, 136, 7)], ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_commit(kind, shape, in_place):
    hk, d, block = shape
    lens = [(5, 40), (0, 9), (1, 1), (300, 320), (64, 64), (7, 100), (3, 3)]
    paths = [[0, 2, 4], [], [0], None, list(range(1, 64)), [], [0, 1, 2]]
    rng = np.random.default_rng(d)
    paths[3] = sorted(rng.choice(300, 170, replace=False).tolist())
    c = P.Case(lens, kind, heads=hk, kv_heads=hk, head_dim=d, block=block, seed=d)
    path = np.full(c.total, -9, np.int32)
    for s, p in enumerate(paths):
        path[c.cu_host[s]:c.cu_host[s] + len(p)] = p
    path, accepted = _dev(path.tolist()), _dev([len(p) for p in paths])
    pos = torch.randint(0, 1000, (len(lens), hk, c.max_kv + 3), dtype=torch.int32, device="cuda", generator=c.g)
    want = [b.raw.clone() for b in c.buffers]
    want_pos = pos.clone()
    for s, ((new, kv), p) in enumerate(zip(lens, paths)):
        slot, off = c.places(s, kv)
        for i, j in enumerate(p):
            a, b = kv - new + j, kv - new + i
            want_pos[s, :, b] = pos[s, :, a]
        for raw, buffer in zip(want, c.buffers):
            other = P.Buffer(kind, c.slots, hk, block, d, c.dtype)
            other.raw = raw
            if not p:
                continue
            came, to = (torch.tensor([kv - new + x for x in q], device="cuda") for q in (p, range(len(p))))
            for name in ("elements",) + (("scales",) if kind == "e4m3" else ()):
                x, y = getattr(buffer, name)(), getattr(other, name)()
                if name == "elements" and kind == "e4m3":
                    x, y = x.view(torch.uint8), y.view(torch.uint8)
                y[slot[to], :, off[to]] = x[slot[came], :, off[came]]
    left = c.kv_len if in_place else torch.full_like(c.kv_len, 77)
    K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), left.data_ptr(), pos=pos.data_ptr(),
                  pos_stride=pos.shape[2], stream=_stream())
    assert left.tolist() == [kv - new + len(p) for (new, kv), p in zip(lens, paths)]
    assert torch.equal(pos, want_pos)
    for b, w in zip(c.buffers, want):
        assert torch.equal(b.raw, w)


def test_commit_beside_absent_blocks_and_wrong_counts():
    """A row from or to an absent block stays; counts outside the new tokens are clamped."""
    c = P.Case([(40, 80), (4, 10), (4, 10)], "16", block=16, absent=[(0, 3)], seed=4)
    before = [b.raw.clone() for b in c.buffers]
    path = _dev(list(range(4, 40)) + [0] * 4 + [1, 2, 3, 3] + [0, 1, 2, 3])
    accepted, left = _dev([36, -3, 99]), _dev([0, 0, 0])
    K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), left.data_ptr(), stream=_stream())
    assert left.tolist() == [76, 6, 10]
    slot, off = c.places(0, 80)
    there = c.there(0, 80)
    for b, was in zip(c.buffers, before):
        old = was.view(torch.bfloat16).view(b.dims)
        for i in range(36):
            source, to = 44 + i, 40 + i
            moved = bool(there[source]) and bool(there[to])
            want = old[slot[source if moved else to], :, off[source if moved else to]]
            assert torch.equal(b.elements()[slot[to], :, off[to]].view(torch.uint8), want.view(torch.uint8))
        slot1, off1 = c.places(1, 10)
        assert torch.equal(b.elements()[slot1, :, off1], old[slot1, :, off1])


# ---- together

@pytest.mark.parametrize("kind", ["e4m3", "16"])
def test_drafts_of_several_steps(kind):
    """Trees appended, attended and committed, step by step: after every commit the cache holds what appending the
    accepted tokens alone would have left, and attention over it is the plain form's."""
    h, hk, d = 8, 2, 64
    room, start = 400, [50, 3, 129]
    c = P.Case([(0, n) for n in start], kind, heads=h, kv_heads=hk, head_dim=d, seed=6, max_kv=room, slots=3 * 26,
               max_q=0)
    rng = np.random.default_rng(6)
    table = _table(room, d)
    lens = list(start)
    full = np.arange(3 * 26).reshape(3, 26).astype(np.int32)     # every sequence has all of its blocks from the start
    for s in range(3):
        used = -(-start[s] // 16)
        full[s, :used] = c.true_table[s, :used]
    taken = set(x for s in range(3) for x in full[s, :-(-start[s] // 16)].tolist())
    free = [x for x in range(3 * 26) if x not in taken]
    for s in range(3):
        for b in range(-(-start[s] // 16), 26):
            full[s, b] = free.pop()
    c.true_table = c.table = np.concatenate([full, np.full((3, c.stride - 26), -7, np.int32)], 1) if c.stride > 26 else full
    c.table_dev, c.stride = _dev(c.table.tolist()), c.table.shape[1]
    twin = [P.Buffer(kind, c.slots, hk, 16, d, c.dtype) for _ in range(2)]
    for a, b in zip(twin, c.buffers):
        a.raw.copy_(b.raw)
    twin_pages = K.Pages(kind, *(b.raw.data_ptr() for b in twin))
    for step in range(3):
        new = [int(x) for x in rng.integers(1, 40, 3)]
        c.lens = [(n, kv + n) for n, kv in zip(new, lens)]
        c.total, c.max_q = sum(new), max(new)
        c.cu_host = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        c.cu, c.kv_len = _dev(c.cu_host.tolist()), _dev([kv for _, kv in c.lens])
        c.batch = K.Batch(3, c.total, c.max_q, room, c.cu.data_ptr(), c.kv_len.data_ptr(), c.table_dev.data_ptr(), c.stride)
        qkv = c.normal(c.total, h + 2 * hk, d)
        bits, mask = c.tree(step, empty=0.0)
        depth = torch.cat([mask[int(c.cu_host[s]):int(c.cu_host[s + 1]), :new[s]].sum(1) - 1 for s in range(3)])
        positions = (depth + torch.cat([torch.full((n,), kv, device="cuda") for n, kv in zip(new, lens)])).int()
        norm = K.HeadNorm(0, 0, 1e-6)
        q = _append(c, qkv, table, d, positions, norm=norm)
        c.read_values()
        _check(_attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))
        # a path down each tree: the ancestors of a token
        path, count = torch.zeros(c.total, dtype=torch.int32), []
        rows = []
        for s in range(3):
            at = int(c.cu_host[s])
            chosen = torch.nonzero(mask[at + int(rng.integers(0, new[s])), :new[s]]).flatten().cpu()
            path[at:at + len(chosen)] = chosen.int()
            count.append(len(chosen))
            rows.append(at + chosen)
        path, accepted = path.cuda(), _dev(count)
        # the twin: the accepted tokens alone
        lens_twin = [kv + n for kv, n in zip(lens, count)]
        cu = np.concatenate([[0], np.cumsum(count)]).tolist()
        cu_dev, len_dev = _dev(cu), _dev(lens_twin)
        rows = torch.cat(rows).cuda()
        few, few_pos = qkv[rows].contiguous(), positions[rows].contiguous()
        batch = K.Batch(3, sum(count), max(count), room, cu_dev.data_ptr(), len_dev.data_ptr(), c.table_dev.data_ptr(), c.stride)
        at, stride = few.data_ptr(), few.stride(0)
        K.norm_rope_append(c.shape, batch, twin_pages, table.data_ptr(), room, d, few_pos.data_ptr(), at + h * d * 2, stride,
                           at + (h + hk) * d * 2, stride, norm=norm, stream=_stream())
        K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), c.kv_len.data_ptr(), stream=_stream())
        assert c.kv_len.tolist() == lens_twin
        lens = lens_twin
        for s in range(3):
            slot, off = c.places(s, lens[s])
            for a, b in zip(c.buffers, twin):
                assert torch.equal(a.rows(slot, off), b.rows(slot, off))
