"""Plain forms in 64 bits of the operators on the paged cache, and the batches that their tests run on."""
import math

import numpy as np
import torch

from paper_2606_14779_amd import kvpool as K

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = {k: torch.finfo(t).eps / 2 for k, t in DTYPE.items()}      # half a unit in the last place, relative
DEV = "cuda"


class Case:
    """A paged cache and a batch over it.  lens: (new, cached) of every sequence.  Slots that no sequence uses, and
    the rows of its last slot past a sequence's end, hold NaN; absent: block table entries replaced by -1 or by a
    slot past the cache."""

    def __init__(self, lens, heads=8, kv_heads=2, head_dim=64, block=16, dtype="bf16", seed=0, absent=(), spare=3,
                 max_q=None, max_kv=None, slots=None, at_end=False):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.heads, self.kv_heads, self.head_dim, self.block, self.dtype = (lens, heads, kv_heads, head_dim,
                                                                                       block, dtype)
        n = len(lens)
        self.max_q = max([q for q, _ in lens] + [0]) if max_q is None else max_q
        self.max_kv = max([kv for _, kv in lens] + [0]) if max_kv is None else max_kv
        self.stride = -(-self.max_kv // block) + 1
        blocks = [-(-kv // block) for _, kv in lens]
        used = sum(blocks)
        self.slots = used + spare if slots is None else slots
        free = np.arange(self.slots)[-used:] if at_end and used else rng.permutation(self.slots)
        table = np.full((n, self.stride), -7, np.int32)
        at = 0
        for i, b in enumerate(blocks):
            table[i, :b] = free[at:at + b]
            at += b
        self.true_table = table.copy()
        for i, (s, b) in enumerate(absent):
            table[s, b] = -1 if i % 2 else self.slots
        self.table = table
        self.total = sum(q for q, _ in lens)
        cu = np.concatenate([[0], np.cumsum([q for q, _ in lens])]).astype(np.int32)
        self.cu_host = cu
        self.g = g

        def dev(a):
            return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        self.cu, self.kv_len = dev(cu), dev(np.array([kv for _, kv in lens], np.int32))
        self.table_dev = dev(table)
        shape = (self.slots, kv_heads, block, head_dim)
        self.k_cache = torch.full(shape, math.nan, dtype=DTYPE[dtype], device=DEV)
        self.v_cache = torch.full(shape, math.nan, dtype=DTYPE[dtype], device=DEV)
        for s, (_, kv) in enumerate(lens):
            if kv:
                slot, off = self.places(s, kv)
                present = dev(np.repeat(table[s] == self.true_table[s], block)[:kv])
                for cache in (self.k_cache, self.v_cache):
                    x = self.normal(kv, kv_heads, head_dim)
                    x[~present] = math.nan              # what an absent slot holds is of no one's concern
                    cache[slot, :, off] = x
        self.shape = K.CacheShape(dtype, heads, kv_heads, head_dim, block, self.slots)
        self.batch = K.Batch(n, self.total, self.max_q, self.max_kv, self.cu.data_ptr(), self.kv_len.data_ptr(),
                             self.table_dev.data_ptr(), self.stride)

    def normal(self, *size, std=1.0, to=None):
        x = torch.empty(size, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=self.g)
        return x.to(DTYPE[self.dtype] if to is None else to)

    def places(self, s, kv):
        slot = torch.from_numpy(np.repeat(self.true_table[s], self.block)[:kv].astype(np.int64)).to(DEV)
        return slot, torch.arange(kv, device=DEV) % self.block

    def there(self, s, kv):
        t = self.table[s]
        return torch.from_numpy(np.repeat((t >= 0) & (t < self.slots), self.block)[:kv]).to(DEV)

    def workspace(self, f):
        n = f(self.shape, self.batch)
        return torch.full((max(n, 16),), 0xA5, dtype=torch.uint8, device=DEV), n


def logits(c, q, s, head, scale, window):
    """64-bit logits of a head's new tokens of sequence s over its cached ones, and which of them each sees."""
    new, kv = c.lens[s]
    slot, off = c.places(s, kv)
    rows = slice(int(c.cu_host[s]), int(c.cu_host[s + 1]))
    kk = c.k_cache[slot, head // (c.heads // c.kv_heads), off].double()
    there = c.there(s, kv)
    kk = torch.where(there[:, None], kk, 0.0)
    z = q[rows, head].double() @ kk.t().contiguous() * scale
    size = q[rows, head].double().abs() @ kk.t().abs().contiguous() * scale
    index = torch.arange(kv - new, kv, device=DEV)[:, None]
    key = torch.arange(kv, device=DEV)[None]
    sees = (key <= index) & there[None]
    if window:
        sees &= key > index - window
    return z, size, sees


def attention(c, q, scale, window=0, sinks=None):
    """(out, lse, tolerance of out, tolerance of lse).

    Tolerances: logits are sums of head_dim products of 16-bit values in 32 bits, off by at most 2^-20 of the sum of
    their magnitudes B; an exponential adds 2^-22; so a weight is off by (2^-20 (B + |lse|) + 2^-21) relative, and
    lse by that and its own rounding.  Weights are rounded to the cache's type (eps each), the output once more.  A
    16-bit float weight below 2^-14 is rounded to a multiple of 2^-24: 2^-25 of the largest value each."""
    out = torch.zeros(c.total, c.heads, c.head_dim, dtype=torch.float64, device=DEV)
    lse = torch.full((c.heads, c.total), -math.inf, dtype=torch.float64, device=DEV)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    eps = EPS[c.dtype]
    for s, (new, kv) in enumerate(c.lens):
        if not new:
            continue
        rows = slice(int(c.cu_host[s]), int(c.cu_host[s + 1]))
        for h in range(c.heads):
            z, size, sees = logits(c, q, s, h, scale, window) if kv else [torch.zeros(new, 0, device=DEV)] * 3
            sees = sees.bool()
            z = torch.where(sees, z.double(), -math.inf)
            size = torch.where(sees, size.double(), 0.0)
            zs = torch.cat([z, sinks[h].double().expand(new, 1)], 1) if sinks is not None else z
            if not zs.shape[1]:
                continue
            e = torch.logsumexp(zs, 1)
            p = torch.where(sees, torch.exp(z - torch.where(e == -math.inf, 0.0, e)[:, None]), 0.0)
            lse[h, rows] = e
            big = size.amax(1) if kv else torch.zeros(new, dtype=torch.float64, device=DEV)
            fe = torch.where(e == -math.inf, 0.0, e).abs()
            rel = 2.0 ** -20 * (big + fe) + 2.0 ** -21 + kv * 2.0 ** -26
            tol_lse[h, rows] = rel + 2.0 ** -22 * fe
            if kv:
                slot, off = c.places(s, kv)
                v = c.v_cache[slot, h // (c.heads // c.kv_heads), off].double()
                v = torch.where(c.there(s, kv)[:, None], v, 0.0)
                o = p @ v
                a = p @ v.abs()
                out[rows, h] = o
                small = 2.0 ** -25 * v.abs().sum(0)[None] if c.dtype == "f16" else 0.0
                tol[rows, h] = (eps + 2 * rel[:, None]) * a + eps * o.abs() + small + 1e-30
                if c.dtype == "f16":
                    tol[rows, h] += 2.0 ** -25
    return out, lse, tol, tol_lse


def mass(c, q, scale, lse, last=0, window=0):
    """(weights [n_seq][kv_heads][max_kv], tolerance): each weight off by 2^-20 (B + |lse|) + 2^-21 relative."""
    out = torch.zeros(len(c.lens), c.kv_heads, c.max_kv, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    for s, (new, kv) in enumerate(c.lens):
        first = max(0, new - last) if last else 0
        if not new or not kv:
            continue
        rows = slice(int(c.cu_host[s]) + first, int(c.cu_host[s + 1]))
        for h in range(c.heads):
            z, size, sees = logits(c, q, s, h, scale, window)
            e = lse[h, rows].double()[:, None]
            sees = sees[first:] & (e > -math.inf)
            p = torch.where(sees, torch.exp(z[first:] - torch.where(e == -math.inf, 0.0, e)), 0.0)
            rel = 2.0 ** -20 * (size[first:] + torch.where(e == -math.inf, 0.0, e).abs()) + 2.0 ** -21
            out[s, h // (c.heads // c.kv_heads), :kv] += p.sum(0)
            tol[s, h // (c.heads // c.kv_heads), :kv] += (p * rel).sum(0) + new * 2.0 ** -26 * p.sum(0)
    return out, tol


def evict(c, keep, protect, score, pos):
    """What is left, by numpy: (source index of every kept place, new lengths)."""
    src, left = {}, []
    for s, (_, kv) in enumerate(c.lens):
        n = min(kv, max(0, keep[s]))
        left.append(n)
        for h in range(c.kv_heads):
            x = score[s, h, :kv].astype(np.float64)
            p = pos[s, h, :kv] if pos is not None else np.arange(kv)
            guarded = p >= protect[s] if protect is not None else np.zeros(kv, bool)
            nan = np.isnan(x) & ~guarded
            order = np.lexsort((np.arange(kv), np.where(guarded | nan, 0.0, -np.where(nan, 0.0, x)), nan, ~guarded))
            kept = order[:n]
            of = np.arange(n)
            of[np.setdiff1d(np.arange(n), kept)] = np.sort(kept[kept >= n])
            src[s, h] = of
    return src, left
