"""``DraftTrees``: trees of drafted tokens over a ``BeamPool`` (speculative decoding of every trace at once).

A round: ``attention`` layer by layer lets every drafted token attend to its beam's context and to its own
ancestors in the beam's tree; the caller picks a path per beam; ``accept`` appends the path's keys and values to the
pool.  The pool does not change until then.  ``BeamPool.truncate`` takes tokens back.

Every operation is one call into ``libgambit.so``; the object keeps the workspace, so its calls belong on one stream.
"""
from __future__ import annotations

import torch

from paper_2608_08020_gb300 import binding as B
from paper_2608_08020_gb300.pool import BeamPool, TORCH_DT


class DraftTrees:
    def __init__(self, pool: BeamPool, n_draft: int):
        self.pool, self.n_draft = pool, n_draft
        c = pool.cfg
        n = B.gb_draft_workspace_bytes(pool.handle, n_draft)
        self.workspace = torch.empty(n, dtype=torch.uint8, device=pool.kv.device)
        if not torch.cuda.is_current_stream_capturing():   # whatever had this memory before is done: calls may be on any stream
            torch.cuda.current_stream(pool.kv.device).synchronize()
        self.device = self.workspace.device
        self._index = self.device.index
        self._args = B.GbDraft(workspace_dev=self.workspace.data_ptr(), workspace_bytes=n, n_draft=n_draft)
        # Whether a round was ever planned here: the library knows a workspace by its address, which an object before this one may
        # have had.
        self._planned = False
        self.dtype = TORCH_DT[pool.kv_dtype]
        self.q_shape = (pool.max_beams, n_draft, c.num_q_heads, c.head_dim)
        self.kv_shape = (pool.max_beams, n_draft, c.num_kv_heads, c.head_dim)
        self._tree_shape, self._slot_shape = self.kv_shape[:2], self.kv_shape[:1]
        self._layers_shape = (c.num_layers, *self.kv_shape)

    def _check(self, name, x, shape, dtype):
        if x.shape != shape or x.dtype is not dtype or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, expected contiguous {shape} {dtype} on "
                             f"{self.device}")
        return x.data_ptr()

    def _draft(self, parent, count):
        d = self._args
        d.parent_dev = self._check("parent", parent, self._tree_shape, torch.int32)
        d.count_dev = None if count is None else self._check("count", count, self._slot_shape, torch.int32)
        return d

    def attention(self, layer: int, q, k, v, parent, scale: float, out=None, count=None, stream=None):
        """One layer: q [max_beams][n_draft][q heads][D], k and v [max_beams][n_draft][kv heads][D], parent int32
        [max_beams][n_draft] (-1: the context's end), count int32 [max_beams] (None: n_draft each); returns out, like q (a new
        one belongs to `stream`, which then has to be a torch.cuda.Stream or None)."""
        if layer > 0 and not self._planned:
            raise B.GambitError(B.GB_ERR_STATE, "draft: layer 0 plans the round")
        if out is None:
            out = torch.empty_like(q) if stream is None else B.new_on(stream, lambda: torch.empty_like(q))
        qs, ks, dt, dev = self.q_shape, self.kv_shape, self.dtype, self._index
        if not (q.shape == qs and k.shape == ks and v.shape == ks and out.shape == qs and q.dtype is dt and k.dtype is dt
                and v.dtype is dt and out.dtype is dt and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
                and out.is_contiguous() and q.get_device() == dev and k.get_device() == dev and v.get_device() == dev
                and out.get_device() == dev):
            for name, x, shape in (("q", q, qs), ("k", k, ks), ("v", v, ks), ("out", out, qs)):
                self._check(name, x, shape, dt)
        B.gb_draft_attention(self.pool.handle, layer, self._draft(parent, count), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                             scale, out.data_ptr(), stream)
        self._planned = self._planned or layer == 0
        return out

    def accept(self, k, v, parent, accepted, count=None, stream=None):
        """Append each slot's path from its tree's root to token accepted[slot] (int32 [max_beams]; -1: none), all
        layers: k and v [layers][max_beams][n_draft][kv heads][D].  Returns (tokens appended int32 [max_beams], their
        indices in order int32 [max_beams][n_draft], then -1)."""
        ka, va = self._check("k", k, self._layers_shape, self.dtype), self._check("v", v, self._layers_shape, self.dtype)
        to = self._check("accepted", accepted, self._slot_shape, torch.int32)
        draft = self._draft(parent, count)
        make = lambda: (torch.empty_like(accepted), torch.empty_like(parent))  # noqa: E731
        n, path = make() if stream is None else B.new_on(stream, make)
        B.gb_accept_draft(self.pool.handle, draft, ka, va, to, n, path, stream)
        return n, path
