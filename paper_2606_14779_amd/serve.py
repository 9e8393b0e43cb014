"""A batch of requests served from the pool, with the operators on the paged cache run as an engine runs them.

A ``ServeRun`` keeps a request per sequence: its context lies offloaded in the pool, comes back into the engine's
paged cache (``kv_pool_retrieve_request``), and then every step of new tokens goes layer by layer through
``kv_rope_append`` (rotated keys and values into the pages), ``kv_attention`` and ``kv_attention_mass`` (the weight
that each cached token collected).  ``evict`` keeps a budget of tokens per head (``kv_evict``), and ``offload``
stores what is left as a new, smaller request.  ``python -m paper_2606_14779_amd.serve`` runs that round trip and
prints what each part took.

There is no model here: the caller hands over each layer's projected queries, keys and values.  All layers have the
same window or none, and no attention sinks, which a caller who needs them passes to ``kvpool.attention`` itself.
"""
from __future__ import annotations

import numpy as np

from . import kvpool as K


class ServeRun:
    """Requests of ``contexts`` tokens each, with room for ``room`` new tokens per sequence.

    shape: anything with layers, kv_heads, head_dim, block_size (``kvgen.workloads.KVShape``); dtype "bf16" or "f16".
    rope: arguments of ``kvpool.rope_table`` past its table, positions and rot_dim.
    """

    def __init__(self, shape, q_heads: int, contexts, room: int, dtype: str = "bf16", window: int = 0, rope=None,
                 device: int = 0, seed: int = 0):
        import torch
        self.torch, self.shape, self.q_heads, self.window = torch, shape, q_heads, window
        self.device = torch.device("cuda", device)
        self.dtype = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
        n, bs = len(contexts), shape.block_size
        self.n = n
        self.max_kv = max(contexts) + room
        self.stride = -(-self.max_kv // bs)
        blocks = [-(-(c + room) // bs) for c in contexts]
        slots = sum(blocks)
        order = np.random.default_rng(seed).permutation(slots).astype(np.int32)
        self.tables, at = [], 0
        table = np.full((n, self.stride), -1, np.int32)
        for i, b in enumerate(blocks):
            self.tables.append(order[at:at + b])
            table[i, :b] = order[at:at + b]
            at += b
        self.slots = slots
        self.most = np.array(contexts, np.int64) + room   # cached tokens that a sequence has room for
        self.table = torch.from_numpy(table).to(self.device)
        self.cache_shape = K.CacheShape(dtype, q_heads, shape.kv_heads, shape.head_dim, bs, slots)
        self.cache, spec = self._new_cache()
        self.k_ptrs = [layer[0].data_ptr() for layer in self.cache]
        self.v_ptrs = [layer[1].data_ptr() for layer in self.cache]
        self.lens = np.array(contexts, np.int32)        # cached tokens
        self.seen = np.array(contexts, np.int64)        # tokens so far: the next one's position
        per_head = (shape.layers, n, shape.kv_heads, self.max_kv)
        self.score = torch.zeros(per_head, dtype=torch.float32, device=self.device)
        self.pos = torch.arange(self.max_kv, dtype=torch.int32, device=self.device).expand(per_head).contiguous()
        self.rot, self.rope = shape.head_dim, dict(rope or {})
        self._positions_up_to(self.max_kv + room)
        held = sum(blocks) * 2 + 2 * n + 2              # twice over, so that a request can be replaced
        self.pool = K.KVPool([K.Region("host", held * spec.block_bytes), K.Region("staging", held * spec.block_bytes)],
                             [1, 1], spec, device)
        self.requests, self._next_request = [None] * n, 1
        self.held = np.zeros(n, bool)                   # whether a sequence's request has its cached tokens as they are
        self._work = None

    def _new_cache(self):
        """The engine's cache, [layers][K and V][slots]..., and its shape for the pool."""
        shape = self.shape
        cache = self.torch.zeros((shape.layers, 2, self.slots, shape.kv_heads, shape.block_size, shape.head_dim),
                                 dtype=self.dtype, device=self.device)
        return cache, K.KVSpec(shape.layers, shape.kv_heads, shape.head_dim, shape.block_size, 2)

    def _stream(self) -> int:
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def _dev(self, a, dtype=None):
        return self.torch.as_tensor(np.ascontiguousarray(a, dtype=dtype or np.int32)).to(self.device)

    def _positions_up_to(self, n: int) -> None:
        """A table of the angles of positions below n."""
        self.n_positions = n
        self.angles = self.torch.empty((n, self.rot // 2, 2), dtype=self.torch.float32, device=self.device)
        with self.torch.cuda.device(self.device):       # the operators launch on the current device
            K.rope_table(self.angles.data_ptr(), n, self.rot, stream=self._stream(), **self.rope)

    def _workspace(self, need: int) -> int:
        if self._work is None or self._work.numel() < need:
            self._work = self.torch.empty(max(need, 16), dtype=self.torch.uint8, device=self.device)
        return self._work.data_ptr()

    # ---- the pool's side
    def offload(self) -> None:
        """Stores every sequence's cached tokens as a request of their own; a request from before is released.  A
        sequence without tokens has none."""
        for i in range(self.n):
            request = None
            blocks = -(-int(self.lens[i]) // self.shape.block_size)
            if blocks:
                request, self._next_request = self._next_request, self._next_request + 1
                loc_map = self.pool.place(request, blocks)
                self.pool.store(loc_map, self.tables[i][:blocks], self.slots, self.k_ptrs, self.v_ptrs, self._stream())
            if self.requests[i] is not None:
                self.pool.release(self.requests[i])
            self.requests[i], self.held[i] = request, True

    def fetch(self) -> None:
        """Brings every sequence's cached tokens back from the pool, where they have not changed since ``offload``."""
        if not self.held.all():
            raise ValueError("sequences %s have changed since they were offloaded" % np.flatnonzero(~self.held).tolist())
        for i in range(self.n):
            blocks = -(-int(self.lens[i]) // self.shape.block_size)
            if blocks:
                self.pool.retrieve_request(self.requests[i], self.tables[i][:blocks], self.slots, self.k_ptrs, self.v_ptrs,
                                           self._stream())

    # ---- the operators' side
    def begin(self, new) -> None:
        """A step of new[i] tokens of sequence i: its lengths and positions, for all layers."""
        new = np.asarray(new, np.int64)
        if len(new) != self.n or (new < 0).any() or (self.lens + new > self.most).any():
            raise ValueError("new tokens do not fit the sequences")
        if (need := int((self.seen + new).max())) > self.n_positions:   # evicted from, a sequence goes on and on
            self._positions_up_to(max(need, 2 * self.n_positions))
        self.lens = (self.lens + new).astype(np.int32)
        cu = np.concatenate([[0], np.cumsum(new)])
        self.total, self.cu, self.kv_len = int(cu[-1]), self._dev(cu), self._dev(self.lens)
        self.positions = self._dev(np.concatenate([np.arange(s, s + k) for s, k in zip(self.seen, new)]))
        self.seen = self.seen + new
        self.held[new > 0] = False
        self.batch = K.Batch(self.n, self.total, int(new.max()), int(self.lens.max()), self.cu.data_ptr(),
                             self.kv_len.data_ptr(), self.table.data_ptr(), self.stride)
        dims = (self.total, self.q_heads, self.shape.head_dim)
        self.q = self.torch.empty(dims, dtype=self.dtype, device=self.device)
        self.lse = self.torch.empty((self.q_heads, self.total), dtype=self.torch.float32, device=self.device)

    def layer(self, index: int, qkv, mass_from: int = 0):
        """Attention output of a layer; qkv [total][q_heads + 2 kv_heads][head_dim] as one projection writes them.
        The weights of the last mass_from new tokens (0: of all) are added to the layer's scores."""
        h, hk, d = self.q_heads, self.shape.kv_heads, self.shape.head_dim
        if tuple(qkv.shape) != (self.total, h + 2 * hk, d) or qkv.dtype != self.dtype or not qkv.is_contiguous():
            raise ValueError("qkv is not [total][q_heads + 2 kv_heads][head_dim] of the cache's type")
        if qkv.device != self.device:
            raise ValueError("qkv is on %s, the cache on %s" % (qkv.device, self.device))
        with self.torch.cuda.device(self.device):
            return self._layer(index, qkv, mass_from)

    def _layer(self, index: int, qkv, mass_from: int):
        h, hk, d = self.q_heads, self.shape.kv_heads, self.shape.head_dim
        stream, row = self._stream(), (h + 2 * hk) * d
        k_cache, v_cache, scale = self.k_ptrs[index], self.v_ptrs[index], d ** -0.5
        at = qkv.data_ptr()
        K.rope_append(self.cache_shape, self.batch, self.angles.data_ptr(), self.n_positions, self.rot,
                      self.positions.data_ptr(), at + h * d * 2, row, at + (h + hk) * d * 2, row, k_cache, v_cache, q=at,
                      q_stride=row, q_out=self.q.data_ptr(), q_out_stride=h * d, pos=self.pos[index].data_ptr(),
                      pos_stride=self.max_kv, stream=stream)
        out = self.torch.empty_like(self.q)
        need = K.attention_workspace(self.cache_shape, self.batch)
        K.attention(self.cache_shape, self.batch, self.q.data_ptr(), h * d, k_cache, v_cache, scale, out.data_ptr(), h * d,
                    window=self.window, lse=self.lse.data_ptr(), workspace=self._workspace(need), workspace_bytes=need,
                    stream=stream)
        score = self.score[index].data_ptr()
        K.attention_mass(self.cache_shape, self.batch, self.q.data_ptr(), h * d, k_cache, scale, self.lse.data_ptr(), score,
                         score, self.max_kv, window=self.window, last=mass_from, stream=stream)
        return out

    def evict(self, keep: int, recent: int) -> None:
        """Keeps `keep` tokens of every sequence, layer and KV head, the `recent` last ones among them.  Not with a
        window: attention counts it in cache indexes, which eviction leaves in no order of positions."""
        if not 0 <= recent <= keep:
            raise ValueError("%d tokens cannot hold the last %d" % (keep, recent))
        if self.window:
            raise ValueError("a windowed cache cannot be evicted from: a window counts cache indexes")
        batch = K.Batch(self.n, 0, 0, int(self.lens.max()), 0, (kv_len := self._dev(self.lens)).data_ptr(),
                        self.table.data_ptr(), self.stride)
        keeps, protect = self._dev(np.full(self.n, keep)), self._dev(self.seen - recent)
        left = self.torch.empty_like(kv_len)
        need = K.evict_workspace(self.cache_shape, batch)
        for i in range(self.shape.layers):
            score, pos = self.score[i].data_ptr(), self.pos[i].data_ptr()
            with self.torch.cuda.device(self.device):
                K.evict(self.cache_shape, batch, keeps.data_ptr(), score, score, self.max_kv, self.k_ptrs[i],
                        self.v_ptrs[i], left.data_ptr(), self._workspace(need), need, protect=protect.data_ptr(),
                        pos_in=pos, pos_out=pos, pos_stride=self.max_kv, stream=self._stream())
        self.held[self.lens > keep] = False
        self.lens = np.minimum(self.lens, keep)

    def close(self) -> None:
        self.pool.close()


def main() -> None:
    import time

    import torch

    from kvgen.workloads import GPT_OSS_20B
    shape, heads, contexts, chunk, keep = GPT_OSS_20B, 64, (32768, 20000, 4097), 256, 2048
    run = ServeRun(shape, heads, contexts, room=512, rope=dict(base=150000.0, kind="by_parts_index", factor=32.0,
                                                               original_length=4096.0, alpha=1.0, beta=32.0))
    for layer in run.cache:
        layer.normal_()

    def timed(what, f):
        torch.cuda.synchronize()
        begin = time.perf_counter()
        f()
        torch.cuda.synchronize()
        print("%-58s %9.2f ms" % (what, 1e3 * (time.perf_counter() - begin)), flush=True)

    def step(new):
        run.begin(new)
        width = (run.total, heads + 2 * shape.kv_heads, shape.head_dim)
        for i in range(shape.layers):
            run.layer(i, torch.randn(width, device=run.device).to(run.dtype), mass_from=32)

    timed("offload %d contexts" % len(contexts), run.offload)
    run.cache.zero_()
    timed("fetch them", run.fetch)
    step([1] * run.n)                                   # kernels are loaded on their first use
    timed("chunks of %d new tokens, %d layers" % (chunk, shape.layers), lambda: step([chunk] * run.n))
    timed("evict to %d tokens a head" % keep, lambda: run.evict(keep, 64))
    timed("offload what is left", run.offload)
    timed("a decoding step", lambda: step([1] * run.n))
    run.close()


if __name__ == "__main__":
    main()
