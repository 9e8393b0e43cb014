"""The operators on pages of either kind and on drafted tokens at the edges of what their header says: batches of very
different lengths and of many sequences, the smallest and largest heads, norms at the ends of the range, caches of more
than 2^32 bytes, device data that is wrong, calls beside each other."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_ops_ref as R   # noqa: E402
import pages_ref as P   # noqa: E402
import test_gpu_pages as T   # noqa: E402
from paper_2606_14779_amd import kvpool as K   # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---- attention

UNEVEN = {
    "one long, many short": [(40, 9000)] + [(3, 10 + i) for i in range(20)] + [(0, 500)],
    "64 sequences": [(1 + i % 33, 40 * i + 40) for i in range(64)],
    "65 sequences": [(1 + i % 33, 40 * i + 40) for i in range(65)],
    "without context": [(100, 100), (1, 1), (0, 0), (65, 65), (33, 4000)],
    "few rows": [(1 + i % 4, 300 * i + 4) for i in range(33)],
    "some rows": [(1 + i % 8, 300 * i + 8) for i in range(33)],
    "more of some": [(1 + i % 16, 211 * i + 16) for i in range(33)],
}


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("lens", list(UNEVEN))
def test_batches_of_different_lengths(kind, window, lens):
    c = P.Case(UNEVEN[lens], kind, heads=8, kv_heads=2, head_dim=64, seed=3)
    q = c.normal(c.total, 8, 64, std=2.0)
    sinks = c.normal(8, to=torch.float32)
    bits, mask = c.tree(1)
    got = T._attend(c, q, 0.125, bits, window, sinks)
    T._check(got, P.attention(c, q, 0.125, window, sinks, mask))
    if kind == "e4m3":
        T._check(T._attend(c, q, 0.125, None, window), P.attention(c, q, 0.125, window))
    for _ in range(3):                               # whatever the order of the workgroups
        again = T._attend(c, q, 0.125, bits, window, sinks)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("shape", [(8, 1, 8, 1), (4, 4, 16, 128), (16, 2, 40, 3), (1, 1, 120, 7), (3, 3, 200, 33), (32, 1, 128, 16)],
                         ids=str)
@pytest.mark.parametrize("new", [1, 4, 20, 50])
def test_heads_and_blocks_of_every_size(shape, new):
    h, hk, d, block = shape
    lens = [(new, 777), (max(1, new // 2), max(1, new // 2)), (new, new + 1)]
    for kind, dtype in (("e4m3", "f16"), ("16", "bf16"), ("e4m3", "bf16")):
        c = P.Case(lens, kind, heads=h, kv_heads=hk, head_dim=d, block=block, dtype=dtype, seed=d, absent=[(0, 0)])
        q = c.normal(c.total, h, d, std=2.0)
        bits, mask = c.tree(new)
        T._check(T._attend(c, q, d ** -0.5, bits), P.attention(c, q, d ** -0.5, mask=mask))


@pytest.mark.parametrize("rows", [4, 24, 48, 200])
def test_logits_in_the_hundreds(rows):
    """A row's largest weight may come late, and others far below it: every rescaling is right."""
    c = P.Case([(rows // 4, 3000), (1, 900)], heads=4, kv_heads=1, head_dim=128, seed=rows)
    q = c.normal(c.total, 4, 128, std=30.0)
    bits, mask = c.tree(2)
    T._check(T._attend(c, q, 1.0, bits), P.attention(c, q, 1.0, mask=mask))


def test_masks_of_more_words_than_a_sequence_has_tokens():
    c = P.Case([(3, 100), (70, 90)], seed=7)
    q = c.normal(c.total, 8, 64)
    for words in (2, 5, 1000):
        bits, mask = c.tree(words, words=words)
        T._check(T._attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))


def test_two_calls_beside_each_other():
    """On two streams, each with its own workspace: what either gives alone."""
    c = P.Case([(24, 6000), (9, 2000), (1, 4000)], heads=8, kv_heads=2, head_dim=128, seed=5)
    q = [c.normal(c.total, 8, 128) for _ in range(2)]
    bits, _ = c.tree(5)
    alone = [T._attend(c, x, 0.1, bits) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [c.workspace(K.attention_pages_workspace)[0] for _ in range(2)]
    outs = [(torch.empty_like(a), torch.empty_like(b)) for a, b in alone]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                T._attend(c, q[i], 0.1, bits, out=outs[i][0], lse=outs[i][1], work=work[i])
    torch.cuda.synchronize()
    for (a, b), (x, y) in zip(alone, outs):
        assert torch.equal(a, x) and torch.equal(b, y)


def test_a_cache_of_16_bits_of_more_than_2_32_bytes():
    slots = (1 << 32) // (2 * 16 * 64 * 2) + 50
    c = P.Case([(30, 600), (1, 70)], "16", heads=8, kv_heads=2, seed=2, slots=slots, at_end=True)
    q = c.normal(c.total, 8, 64)
    bits, mask = c.tree(2)
    T._check(T._attend(c, q, 0.125, bits), P.attention(c, q, 0.125, mask=mask))
    # and accepted drafts move where they are
    slot, off = c.places(0, 600)
    want = [b.rows(slot[[572, 580, 599]], off[[572, 580, 599]]) for b in c.buffers]
    path, accepted, left = T._dev([2, 10, 29] + [0] * 28), T._dev([3, 0]), T._dev([0, 0])
    K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), left.data_ptr(), stream=T._stream())
    assert left.tolist() == [573, 69]
    for b, w in zip(c.buffers, want):
        assert torch.equal(b.rows(slot[570:573], off[570:573]), w)


def test_lengths_that_are_too_long_are_cut():
    """Lengths in device memory past what the batch says: as if they were what it says."""
    c = P.Case([(5, 100), (9, 64)], seed=8, max_kv=100)
    q = c.normal(c.total, 8, 64)
    bits, mask = c.tree(8)
    want = P.attention(c, q, 0.125, mask=mask)
    c.kv_len[0] = 1 << 29
    T._check(T._attend(c, q, 0.125, bits), want)
    path, accepted, left = T._dev([-7, 1 << 30, 2, 3, 4] + [0] * 9), T._dev([5, 1 << 30]), T._dev([0, 0])
    K.tree_commit(c.shape, c.batch, c.pages, path.data_ptr(), accepted.data_ptr(), left.data_ptr(), stream=T._stream())
    assert left.tolist() == [100, 64]


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("lens", [[(2, 5000), (1, 900)], [(12, 6000), (0, 40), (3, 10)], [(200, 9000), (7, 7)], [(3, 20)]])
def test_rows_behind_the_last_sequence(kind, lens):
    """A batch padded to more tokens than its sequences have: the others as without, the rows behind as they were."""
    c = P.Case(lens, kind, heads=8, kv_heads=2, head_dim=64, seed=len(lens))
    q = c.normal(c.total + 5, 8, 64)
    bits, _ = c.tree(1)
    tail = torch.full((5, bits.shape[1]), -1, dtype=torch.int64, device="cuda")
    plain, real = c.batch, c.total
    padded = K.Batch(len(lens), real + 5, c.max_q, c.max_kv, c.cu.data_ptr(), c.kv_len.data_ptr(), c.table_dev.data_ptr(),
                     c.stride)
    qkv, positions = c.normal(real + 5, 12, 64), torch.zeros(real + 5, dtype=torch.int32, device="cuda")
    for tree in (None, bits):
        c.batch, c.total = plain, real
        want = P.attention(c, q[:real], 0.125, mask=c.tree(1)[1] if tree is not None else None)
        c.batch, c.total = padded, real + 5
        out, lse = T._attend(c, q, 0.125, torch.cat([tree, tail]) if tree is not None else None)
        T._check((out[:real], lse[:, :real]), want)
        assert (out[real:] == 7).all() and (lse[:, real:] == 7).all()
    before = [b.raw.clone() for b in c.buffers]
    q_out = T._append(c, qkv, T._table(1, 64), 64, positions)
    assert (q_out[real:] == 3).all() and not (q_out[:real] == 3).all((1, 2)).any()
    # nothing but the new tokens' rows was written
    for b, old in zip(c.buffers, before):
        got = b.raw.clone()
        b.raw.copy_(old)
        c.batch, c.total = plain, real
        T._append(c, qkv[:real], T._table(1, 64), 64, positions[:real])
        assert torch.equal(got, b.raw)
        b.raw.copy_(got)


# ---- append

@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("n", [64, 65, 700])
def test_append_to_many_sequences(kind, n):
    """Every token to its own sequence's pages, whichever of them have none."""
    rng = np.random.default_rng(n)
    lens = [(int(q), int(q + rng.integers(0, 40))) for q in rng.integers(0, 3, n)]
    c = P.Case(lens, kind, heads=4, kv_heads=2, head_dim=32, seed=n)
    qkv = c.normal(c.total, 8, 32)
    positions = torch.randint(0, 90, (1, c.total), dtype=torch.int32, device="cuda", generator=c.g)
    pos = torch.full((n, 2, c.max_kv), -1, dtype=torch.int32, device="cuda")
    T._append(c, qkv, T._table(90, 32), 32, positions, pos=pos)
    for s, (new, kv) in enumerate(lens):
        if not new:
            continue
        rows = slice(int(c.cu_host[s]), int(c.cu_host[s + 1]))
        slot, off = (x[kv - new:] for x in c.places(s, kv))
        other = P.Buffer(kind, c.slots, 2, 16, 32, c.dtype)
        other.put(slot, off, qkv[rows, 6:8])
        assert torch.equal(c.buffers[1].rows(slot, off), other.rows(slot, off))
        assert torch.equal(pos[s, :, kv - new:kv], positions[:, rows].expand(2, -1))


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (120, True), (0, False), (124, False)])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
def test_norms_of_the_smallest_and_largest_heads(rot, interleaved, eps):
    """bf16 from its subnormal numbers to its largest: mean squares from 2^-266 to 2^256, weighted."""
    c = P.Case([(12, 12)], "16", heads=1, kv_heads=1, head_dim=128, seed=1)
    x = c.normal(12, 128, to=torch.float64)
    x = x / x.abs().amax(1, keepdim=True)
    x *= P.pow2(torch.tensor([127, 126, 100, 64, 59, 1, -49, -51, -64, -100, -125, -132], device="cuda"))[:, None]
    qkv = x.to(torch.bfloat16)[:, None].expand(12, 3, 128).contiguous()
    positions, table = torch.arange(12, dtype=torch.int32, device="cuda")[None], T._table(12, rot)
    w = c.normal(128)
    q_out = T._append(c, qkv, table, rot, positions, norm=K.HeadNorm(w.data_ptr(), 0, eps), interleaved=interleaved)
    want, err = P.turned(qkv[:, :1], w, eps, table, positions, [0] * 64, rot, interleaved, True)
    # what is smaller than 32 bits hold (2^-149) at any stage is gone
    assert T._near(q_out, want, err + 2.0 ** -126, "bf16")
    keys = c.buffers[0].rows(*c.places(0, 12))
    want, err = P.turned(qkv[:, 1:2], None, eps, table, positions, [0] * 64, rot, interleaved, True)
    assert T._near(keys, want, err + 2.0 ** -126, "bf16")


@pytest.mark.parametrize("rot,interleaved", [(0, False), (128, True), (64, False), (12, False)])
def test_norms_with_the_smallest_and_largest_weights(rot, interleaved):
    """Heads of any size times weights from 2^-120 to 2^120: only the product with the normed head has to fit."""
    c = P.Case([(9, 9)], "16", heads=1, kv_heads=1, head_dim=128, seed=2)
    x = c.normal(9, 128, to=torch.float64)
    x = x / x.abs().amax(1, keepdim=True) * P.pow2(torch.tensor([120, 58, 50, 20, 0, -20, -40, -48, -120], device="cuda"))[:, None]
    qkv = x.to(torch.bfloat16)[:, None].expand(9, 3, 128).contiguous()
    positions, table = torch.arange(9, dtype=torch.int32, device="cuda")[None], T._table(9, rot)
    w = (1.5 * P.pow2(torch.arange(128, device="cuda") // 32 * 80 - 120)).to(torch.bfloat16)     # pairs of unlike weights
    q_out = T._append(c, qkv, table, rot, positions, norm=K.HeadNorm(w.data_ptr(), w.data_ptr(), 0.0), interleaved=interleaved)
    want, err = P.turned(qkv[:, :1], w, 0.0, table, positions, [0] * 64, rot, interleaved, True)
    assert T._near(q_out, want, err + 2.0 ** -126, "bf16")
    assert T._near(c.buffers[0].rows(*c.places(0, 9)), want, err + 2.0 ** -126, "bf16")


def test_rows_of_128_elements_with_what_is_no_number():
    """Infinities and NaN cost the 32 elements they are among nothing but themselves."""
    c = P.Case([(40, 40)], heads=1, kv_heads=1, head_dim=128, seed=4)
    x = c.normal(40, 128)
    for i in range(40):
        x[i, 3 * i] = [math.inf, -math.inf, math.nan][i % 3]
    qkv = x[:, None].expand(40, 3, 128).contiguous()
    T._append(c, qkv, T._table(1, 0), 0, torch.zeros(40, dtype=torch.int32, device="cuda"), q=False)
    want, e = P.pack(x, "bf16")
    slot, off = c.places(0, 40)
    for b in c.buffers:
        got = b.elements()[slot, 0, off].float()
        assert torch.equal(got.nan_to_num(999.0), want.float().nan_to_num(999.0))
        assert torch.equal(b.scales()[slot, 0, off], e)


# ---- conversion

@pytest.mark.parametrize("back", [False, True])
def test_convert_caches_of_more_than_2_32_bytes(back):
    slots = (1 << 32) // (2 * 16 * (68 if back else 128)) + 20
    a, b = ("e4m3", "16") if back else ("16", "e4m3")
    c = P.Case([(0, 300), (0, 40)], a, heads=2, kv_heads=2, head_dim=64, seed=6, slots=slots, at_end=True)
    to = [P.Buffer(b, slots, 2, 16, 64, c.dtype) for _ in range(2)]
    K.convert_pages(c.shape, c.batch, c.pages, K.Pages(b, *(x.raw.data_ptr() for x in to)), c.table_dev.data_ptr(), c.stride,
                    slots, stream=T._stream())
    for s, (_, kv) in enumerate(c.lens):
        slot, off = c.places(s, kv)
        for source, out in zip(c.buffers, to):
            rows = source.rows(slot, off)
            if back:
                assert torch.equal(out.rows(slot, off), rows)
            else:
                y, e = P.pack(rows, c.dtype)
                assert torch.equal(out.rows(slot, off), P.unpack(y, e))


def test_convert_many_sequences():
    rng = np.random.default_rng(2)
    lens = [(0, int(x)) for x in rng.integers(0, 200, 500)]
    c = P.Case(lens, "e4m3", heads=2, kv_heads=2, head_dim=80, block=8, seed=9)
    to = [P.Buffer("16", c.slots, 2, 8, 80, c.dtype) for _ in range(2)]
    K.convert_pages(c.shape, c.batch, c.pages, K.Pages("16", *(x.raw.data_ptr() for x in to)), c.table_dev.data_ptr(), c.stride,
                    c.slots, stream=T._stream())
    for s, (_, kv) in enumerate(lens):
        if kv:
            slot, off = c.places(s, kv)
            for source, out in zip(c.buffers, to):
                assert torch.equal(out.rows(slot, off), source.rows(slot, off))


@pytest.mark.parametrize("kind", ["e4m3", "16"])
@pytest.mark.parametrize("window", [1, 128, 1000])
def test_a_large_windowed_tree(kind, window):
    """Row tiles that all go over the window and every draft, in parts."""
    c = P.Case([(1500, 4000)], kind, heads=4, kv_heads=1, head_dim=128, seed=window)
    q = c.normal(c.total, 4, 128, std=2.0)
    bits, mask = c.tree(window)
    T._check(T._attend(c, q, 128 ** -0.5, bits, window), P.attention(c, q, 128 ** -0.5, window, mask=mask))
