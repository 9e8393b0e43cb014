"""A batch of requests served from the pool over pages of either kind, with drafted tokens checked several at a time.

A ``DraftRun`` is a ``ServeRun`` whose engine cache is 8-bit pages (or 16-bit ones): the pool moves half the bytes.  A
step's new tokens go layer by layer through ``kv_norm_rope_append`` (queries and keys normed where the model does so,
turned, and written to the pages) and ``kv_attention_pages``.  New tokens may be drafts that form a tree: each sees the
context and its own ancestors, as far as a window lets it, and after the caller has checked them, ``commit`` keeps a path
of each tree (``kv_tree_commit``) and the others are gone.  ``python -m paper_2606_14779_amd.drafts`` runs that and prints what each
part took.
"""
from __future__ import annotations

import numpy as np

from . import kvpool as K
from .serve import ServeRun


def tree_mask(parents) -> np.ndarray:
    """Rows of 64-bit words for the drafts of one sequence: token i sees itself and its ancestors.  parents[i] is the
    draft before it, less than i, or -1."""
    n = len(parents)
    sees = np.zeros((n, max(1, -(-n // 64)) * 64), bool)
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError("the parent of draft %d is %d" % (i, p))
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return np.packbits(sees, axis=1, bitorder="little").view(np.int64)


def _within(bits, depth, window: int):
    """What the drafts of one sequence see under a window: of a mask [drafts][bits], whose draft i stands depth[i] places
    behind the first, the ones less than `window` places before a draft.  ``kv_attention_pages`` finds a draft's place in
    the window by how many drafts it sees: all before it that are near enough to hide what is cached must be there."""
    n = len(depth)
    near = bits.copy()
    near[:, :n] &= (depth[:, None] - depth[None, :] < window).astype(bits.dtype)
    count = near[:, :n].sum(1, dtype=np.int64)
    if (count < np.minimum(depth + 1, window)).any():
        raise ValueError("a draft that does not see the %d drafts before it that a window leaves" % (window - 1))
    return near


class DraftRun(ServeRun):
    """Arguments as of ``ServeRun``, and

    pages: "e4m3" or "16".
    norm: None, or (weights of the queries' norm, of the keys', eps); weights [layers][head_dim] of the cache's type.

    No scores of attention mass are collected, so there is no eviction.
    """

    def __init__(self, shape, q_heads: int, contexts, room: int, dtype: str = "bf16", pages: str = "e4m3", norm=None, **kw):
        self.kind = pages
        self.drafted = None                             # new tokens of every sequence that wait for commit
        self.batch = None                               # of the step that layers are run for
        super().__init__(shape, q_heads, contexts, room, dtype, **kw)
        self.pages = [K.Pages(pages, k, v) for k, v in zip(self.k_ptrs, self.v_ptrs)]
        self.norm = None
        if norm is not None:
            for w in norm[:2]:
                if tuple(w.shape) != (shape.layers, shape.head_dim) or w.dtype != self.dtype or not w.is_contiguous() \
                        or w.device != self.device:
                    raise ValueError("a norm's weights are not [layers][head_dim] of the cache's type on %s" % self.device)
            # rows begin at 16 bytes: head_dim is a multiple of 8
            self._norm_weights = norm[:2]
            self.norm = [K.HeadNorm(q.data_ptr(), k.data_ptr(), norm[2]) for q, k in zip(*norm[:2])]

    def _new_cache(self):
        if self.kind == "16":
            return super()._new_cache()
        shape, slot = self.shape, K.page_bytes(self.cache_shape, self.kind)
        rows = shape.kv_heads * shape.block_size
        if slot % rows:
            raise ValueError("%d bytes of a slot are no whole bytes of its %d rows" % (slot, rows))
        cache = self.torch.zeros((shape.layers, 2, self.slots, slot), dtype=self.torch.uint8, device=self.device)
        return cache, K.KVSpec(shape.layers, shape.kv_heads, slot // rows, shape.block_size, 1)

    def _settled(self) -> None:
        if self.drafted is not None:
            raise ValueError("drafted tokens wait for commit")

    def offload(self) -> None:
        self._settled()
        super().offload()

    def fetch(self) -> None:
        self._settled()
        super().fetch()

    def evict(self, keep: int, recent: int) -> None:
        raise ValueError("no scores to evict by: attention mass is not collected here")

    def begin(self, new, tree=None) -> None:
        """A step of new[i] tokens of sequence i; tree: None, or the rows of ``tree_mask`` of all sequences, one after the
        other, all of the same number of words.  A draft's place behind the cached tokens is the number of drafts before it
        that its row has; under a window it sees none of those that are `window` or more places before it."""
        self._settled()
        new, seen = np.asarray(new, np.int64), self.seen
        if tree is not None:
            tree = np.ascontiguousarray(tree, dtype=np.int64)
            if tree.ndim != 2 or tree.shape[0] != new.sum() or tree.shape[1] * 64 < new.max(initial=0):
                raise ValueError("tree is not [new tokens][words]")
            bits = np.unpackbits(tree.view(np.uint8), axis=1, bitorder="little")
            sees = [bits[a:a + n, :n].astype(bool) for a, n in zip(np.cumsum(new) - new, new)]
            depth = [x.sum(1, dtype=np.int64) - 1 for x in sees]
            if any((d < 0).any() for d in depth):
                raise ValueError("a draft that sees no draft, not even itself")
            if self.window:
                near = [_within(bits[a:a + n], d, self.window) for a, n, d in zip(np.cumsum(new) - new, new, depth)]
                tree = np.packbits(np.concatenate(near), axis=1, bitorder="little").view(np.int64)
        super().begin(new)
        self.tree = None
        if tree is not None:
            self.positions = self._dev(np.concatenate([s + d for s, d in zip(seen, depth)]))
            self.tree, self.drafted, self.seen = self._dev(tree, np.int64), new, seen
            self._sees = sees                           # which drafts of its sequence each one follows

    def layer(self, index: int, qkv, mass_from: int = 0):
        """Attention output of a layer; qkv as in ``ServeRun.layer``."""
        if mass_from:
            raise ValueError("attention mass is not collected here")
        if self.batch is None:
            raise ValueError("no step has begun")
        return super().layer(index, qkv)

    def _layer(self, index: int, qkv, mass_from: int):
        h, hk, d = self.q_heads, self.shape.kv_heads, self.shape.head_dim
        stream, row, at = self._stream(), (h + 2 * hk) * d, qkv.data_ptr()
        K.norm_rope_append(self.cache_shape, self.batch, self.pages[index], self.angles.data_ptr(), self.n_positions, self.rot,
                           self.positions.data_ptr(), at + h * d * 2, row, at + (h + hk) * d * 2, row,
                           norm=self.norm[index] if self.norm else None, q=at, q_stride=row, q_out=self.q.data_ptr(),
                           q_out_stride=h * d, pos=self.pos[index].data_ptr(), pos_stride=self.max_kv, stream=stream)
        tree = self.tree if self.total else None        # a step without tokens has no rows to point to
        out = self.torch.empty_like(self.q)
        need = K.attention_pages_workspace(self.cache_shape, self.batch)
        K.attention_pages(self.cache_shape, self.batch, self.pages[index], self.q.data_ptr(), h * d, d ** -0.5,
                          out.data_ptr(), h * d, tree=tree.data_ptr() if tree is not None else 0,
                          tree_words=tree.shape[1] if tree is not None else 0, window=self.window,
                          lse=self.lse.data_ptr(), workspace=self._workspace(need), workspace_bytes=need, stream=stream)
        return out

    def commit(self, paths) -> None:
        """paths[i]: the accepted drafts of sequence i, ascending as a path down its tree is: each of them sees those before
        it, and none that is not accepted."""
        if self.drafted is None:
            raise ValueError("no drafted tokens")
        paths = [np.asarray(p, np.int64).reshape(-1) for p in paths]
        if len(paths) != self.n:
            raise ValueError("one path per sequence")
        for p, n, sees in zip(paths, self.drafted, self._sees):
            if len(p) and (p[0] < 0 or p[-1] >= n or (np.diff(p) <= 0).any()):
                raise ValueError("a path is not ascending among its sequence's %d drafts" % n)
            # one left out, or one of another branch, would leave positions with holes and outputs of other contexts
            if np.delete(sees[p], p, axis=1).any() or not sees[np.ix_(p, p)][np.tril_indices(len(p))].all():
                raise ValueError("drafts %s are no path of their sequence's tree from its first on" % p.tolist())
        path = np.zeros(max(self.total, 1), np.int32)
        for a, p in zip(np.cumsum(self.drafted) - self.drafted, paths):
            path[a:a + len(p)] = p
        count = np.array([len(p) for p in paths], np.int64)
        path, accepted, left = self._dev(path), self._dev(count), self.torch.empty_like(self.kv_len)
        with self.torch.cuda.device(self.device):
            for i in range(self.shape.layers):
                K.tree_commit(self.cache_shape, self.batch, self.pages[i], path.data_ptr(), accepted.data_ptr(),
                              left.data_ptr(), pos=self.pos[i].data_ptr(), pos_stride=self.max_kv, stream=self._stream())
        self.lens = (self.lens - self.drafted + count).astype(np.int32)
        self.seen = self.seen + count
        self.kv_len, self.drafted = left, None
        self.batch = None                               # whose lengths were those before


def main() -> None:
    import dataclasses
    import time

    import torch

    from kvgen.workloads import QWEN3_30B_A3B
    shape, heads, contexts, drafts = QWEN3_30B_A3B, 32, (32768, 20000, 4097), 16
    rng = np.random.default_rng(0)
    one = torch.ones((shape.layers, shape.head_dim), dtype=torch.bfloat16, device="cuda")

    for kind, block in (("16", 16), ("e4m3", 64)):      # slots of 16 and 33 KB
        run = DraftRun(dataclasses.replace(shape, block_size=block), heads, contexts, room=512, pages=kind,
                       norm=(one, one, 1e-6), rope=dict(base=1000000.0))

        def timed(what, f):
            torch.cuda.synchronize()
            begin = time.perf_counter()
            f()
            torch.cuda.synchronize()
            took = 1e3 * (time.perf_counter() - begin)
            print("%-58s %9.2f ms" % ("%s bits: %s" % (kind if kind == "16" else "8", what), took), flush=True)

        def step(new, tree=None):
            run.begin(new, tree)
            width = (run.total, heads + 2 * shape.kv_heads, shape.head_dim)
            for i in range(shape.layers):
                run.layer(i, torch.randn(width, device=run.device).to(run.dtype))

        def drafted():
            parents = [[-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, drafts)] for _ in contexts]
            step([drafts] * run.n, np.concatenate([tree_mask(p) for p in parents]))
            paths = []
            for p in parents:
                path, at = [], drafts - 1
                while at >= 0:
                    path.append(at)
                    at = p[at]
                paths.append(path[::-1])
            run.commit(paths)

        timed("offload %d contexts" % len(contexts), run.offload)
        timed("fetch them", run.fetch)
        drafted()                                       # kernels are loaded on their first use
        timed("%d drafts each, %d layers, checked and committed" % (drafts, shape.layers), drafted)
        step([1] * run.n)
        timed("a decoding step", lambda: step([1] * run.n))
        run.close()


if __name__ == "__main__":
    main()
