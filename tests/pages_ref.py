"""Plain forms in 64 bits of the operators on pages of either kind and on drafted tokens, and pages that their tests run
on."""
import math

import numpy as np
import torch

import cache_ops_ref as R
from paper_2606_14779_amd import kvpool as K

LIMITS = {"bf16": (-117, 120), "f16": (-15, 8)}      # exponents


def row_exponents(d):
    return 4 * -(-d // 128)


def pow2(e):
    """2^e of whole numbers in 64 bits, exactly."""
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def exponents(x, dtype):
    """The least e with max |x| <= 448 * 2^e for 32 elements each (finite ones), within the type's limits."""
    d = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    least, most = LIMITS[dtype]
    e = torch.full(top.shape, least, dtype=torch.int32, device=x.device)
    for i in range(least, most):
        e += (top > 448.0 * 2.0 ** i).int()
    return e


def pack(x, dtype):
    """(elements, bytes of exponents) of rows, as e4m3 and uint8 of row_exponents."""
    d = x.shape[-1]
    e = exponents(x, dtype)
    power = pow2(e).repeat_interleave(32, -1)[..., :d]
    limit = torch.where(e == LIMITS[dtype][1], 240.0, 448.0).double().repeat_interleave(32, -1)[..., :d]
    y = x.double() / power
    y = torch.where(torch.isfinite(y), torch.maximum(torch.minimum(y, limit), -limit), math.nan)
    # values of at most 24 bits after the division by a power of two: 32 bits hold them
    out = y.float().to(torch.float8_e4m3fn)
    return out, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, row_exponents(d) - e.shape[-1]))


def unpack(x, e):
    d = x.shape[-1]
    power = pow2(e.int() - 127).repeat_interleave(32, -1)[..., :d]
    return x.double() * power


class Buffer:
    """A K or V buffer of one kind: bytes of slots, all of them other than 0 at first."""

    def __init__(self, kind, slots, kv_heads, block, d, dtype):
        self.kind, self.dims, self.dtype = kind, (slots, kv_heads, block, d), dtype
        shape = K.CacheShape(dtype, kv_heads, kv_heads, d, block, slots)
        self.slot = K.page_bytes(shape, kind)
        self.raw = torch.full((slots, self.slot), 0x7F, dtype=torch.uint8, device=R.DEV)   # NaN in either kind, or nearly

    def elements(self):
        slots, hk, bs, d = self.dims
        n = hk * bs * d
        if self.kind == "16":
            return self.raw.view(R.DTYPE[self.dtype]).view(slots, hk, bs, d)
        return self.raw[:, :n].view(slots, hk, bs, d).view(torch.float8_e4m3fn)

    def scales(self):
        slots, hk, bs, d = self.dims
        n, e = hk * bs * d, row_exponents(d)
        return self.raw[:, n:n + hk * bs * e].view(slots, hk, bs, e)

    def put(self, slot, off, x):
        """Rows [tokens][kv_heads][d]."""
        if self.kind == "16":
            self.elements()[slot, :, off] = x.to(R.DTYPE[self.dtype])
        else:
            y, e = pack(x, self.dtype)
            self.elements().view(torch.uint8)[slot, :, off] = y.view(torch.uint8)
            self.scales()[slot, :, off] = e

    def rows(self, slot, off):
        """Rows [tokens][kv_heads][d] in 64 bits."""
        if self.kind == "16":
            return self.elements()[slot, :, off].double()
        x = self.elements().view(torch.uint8)[slot, :, off].view(torch.float8_e4m3fn)
        return unpack(x, self.scales()[slot, :, off])


class Case(R.Case):
    """A batch whose cache is pages of a kind.  k_cache and v_cache hold the values that the pages stand for, NaN
    where no sequence has a token."""

    def __init__(self, lens, kind="e4m3", **kw):
        super().__init__(lens, **kw)
        self.kind = kind
        self.buffers = []
        for name in ("k_cache", "v_cache"):
            b = Buffer(kind, self.slots, self.kv_heads, self.block, self.head_dim, self.dtype)
            for s, (_, kv) in enumerate(lens):
                if kv:
                    slot, off = self.places(s, kv)
                    b.put(slot, off, getattr(self, name)[slot, :, off])
            self.buffers.append(b)
        self.pages = K.Pages(kind, *(b.raw.data_ptr() for b in self.buffers))
        self.read_values()

    def read_values(self):
        for name, b in zip(("k_cache", "v_cache"), self.buffers):
            cache = torch.full(b.dims, math.nan, dtype=R.DTYPE[self.dtype], device=R.DEV)
            for s, (_, kv) in enumerate(self.lens):
                if kv:
                    slot, off = self.places(s, kv)
                    cache[slot, :, off] = b.rows(slot, off).to(R.DTYPE[self.dtype])   # exact
            setattr(self, name, cache)

    def tree(self, seed, empty=0.1, words=None):
        """A mask [total][words] as 64-bit words and [total][max_q] as truth values: a tree, some rows of which see
        nothing new, and bits past a sequence's new tokens set at random."""
        rng = np.random.default_rng(seed)
        words = max(1, -(-self.max_q // 64)) if words is None else words
        mask = np.zeros((self.total, words * 64), bool)
        for s, (new, _) in enumerate(self.lens):
            at = int(self.cu_host[s])
            for i in range(new):
                p = int(rng.integers(max(0, i - 4), i)) if i and rng.random() < 0.9 else -1
                if p >= 0:
                    mask[at + i] |= mask[at + p]
                mask[at + i, i] = True
            for i in range(new):
                if rng.random() < empty:
                    mask[at + i] = False
            mask[at:at + new, new:] = rng.random((new, words * 64 - new)) < 0.5
        bits = np.packbits(mask, axis=1, bitorder="little").view(np.int64)
        return torch.from_numpy(bits.copy()).to(R.DEV), torch.from_numpy(mask).to(R.DEV)


def sees(c, s, window, mask):
    """Which cached tokens each new one of sequence s sees."""
    new, kv = c.lens[s]
    first = kv - new
    key = torch.arange(kv, device=R.DEV)[None]
    i = torch.arange(new, device=R.DEV)[:, None]
    if mask is None:
        out = key <= first + i
        if window:
            out &= key > first + i - window
    else:
        mine = mask[int(c.cu_host[s]):int(c.cu_host[s + 1]), :new]
        out = (key < first).repeat(new, 1)
        if window:
            out &= key > first + mine.sum(1, keepdim=True) - 1 - window
        out[:, first:] = mine
    return out & c.there(s, kv)[None]


def attention(c, q, scale, window=0, sinks=None, mask=None):
    """(out, lse, tolerance of out, tolerance of lse), as cache_ops_ref.attention derives them: elements of 8 bits are
    exact in the type that products are made of."""
    out = torch.zeros(c.total, c.heads, c.head_dim, dtype=torch.float64, device=R.DEV)
    lse = torch.full((c.heads, c.total), -math.inf, dtype=torch.float64, device=R.DEV)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    eps, group = R.EPS[c.dtype], c.heads // c.kv_heads
    for s, (new, kv) in enumerate(c.lens):
        if not new:
            continue
        rows = slice(int(c.cu_host[s]), int(c.cu_host[s + 1]))
        seen = sees(c, s, window, mask)
        slot, off = c.places(s, kv)
        there = c.there(s, kv)[:, None, None]
        k = torch.where(there, c.k_cache[slot, :, off].double(), 0.0)
        v = torch.where(there, c.v_cache[slot, :, off].double(), 0.0)
        for h in range(c.heads):
            qq, kk, vv = q[rows, h].double(), k[:, h // group].contiguous(), v[:, h // group].contiguous()
            z = torch.where(seen, qq @ kk.t().contiguous() * scale, -math.inf)
            big = torch.where(seen, qq.abs() @ kk.t().abs().contiguous() * scale, 0.0).amax(1)
            zs = torch.cat([z, sinks[h].double().expand(new, 1)], 1) if sinks is not None else z
            e = torch.logsumexp(zs, 1)
            fe = torch.where(e == -math.inf, 0.0, e)
            p = torch.where(seen, torch.exp(z - fe[:, None]), 0.0)
            lse[h, rows] = e
            rel = 2.0 ** -20 * (big + fe.abs()) + 2.0 ** -21 + kv * 2.0 ** -26
            tol_lse[h, rows] = rel + 2.0 ** -22 * fe.abs()
            o, a = p @ vv, p @ vv.abs()
            out[rows, h] = o
            small = 2.0 ** -25 * vv.abs().sum(0)[None] + 2.0 ** -25 if c.dtype == "f16" else 0.0
            tol[rows, h] = (eps + 2 * rel[:, None]) * a + eps * o.abs() + small + 1e-30
    return out, lse, tol, tol_lse


def turned(x, weight, eps, table, positions, axis_of, rot, interleaved, norm):
    """(value, error of 32 bits) of heads [tokens][heads][d] normed and turned.

    The factor of the norm: 13 roundings of a sum of squares, two of the mean with eps, halved by the root, and two units of
    the root: 10 * 2^-24; two products and two roundings of the turn: 14 * 2^-24 of the turned magnitudes, below 2^-20."""
    x = x.double()
    if norm:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * (weight.double() if weight is not None else 1.0)
    out, size = x.clone(), x.abs()
    half = rot // 2
    if half:
        first = list(range(0, rot, 2)) if interleaved else list(range(half))
        second = [i + 1 for i in first] if interleaved else [i + half for i in first]
        pair = torch.arange(half, device=x.device)
        where = positions.long()[torch.tensor(axis_of, device=x.device)[:half]].t()          # [tokens][pairs]
        cos, sin = table.double()[where, pair].unbind(-1)
        cos, sin = cos[:, None], sin[:, None]
        a, b = x[..., first], x[..., second]
        out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
        size[..., first] = (a * cos).abs() + (b * sin).abs()
        size[..., second] = (b * cos).abs() + (a * sin).abs()
    return out, size * 2.0 ** -20
