"""``PromptAttention``: causal attention over whole prompts, packed one after the other.

The prefill beside the beam pool: it computes the prompt's own attention, layer by layer, whose keys and
values ``BeamPool.seed`` then takes (Algorithm 1, "S <- C initial traces from P").  Each call is one call of
``gb_prompt_attention``; the object keeps the workspace, so calls of one object belong on one stream.
"""
from __future__ import annotations

import torch

from paper_2608_08020_gb300 import binding as B
from paper_2608_08020_gb300.pool import _DT, TORCH_DT


class PromptAttention:
    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, dtype: str, *, max_tokens: int, max_seqs: int,
                 device: str | torch.device = "cuda"):
        self.num_q_heads, self.num_kv_heads, self.head_dim, self.dtype = num_q_heads, num_kv_heads, head_dim, dtype
        self.max_tokens, self.max_seqs, self.device = max_tokens, max_seqs, torch.device(device)
        n = B.gb_prompt_workspace_bytes(max_tokens, max_seqs, num_q_heads, num_kv_heads, head_dim, _DT[dtype])
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=self.device)

    def __call__(self, q, k, v, cu_seqlens, scale: float, out=None, stream=None):
        """q [tokens][q heads][head_dim], k and v [tokens][kv heads][head_dim] (each token's heads contiguous, tokens
        at any stride), cu_seqlens int32 [seqs + 1]; returns out [tokens][q heads][head_dim] (new unless given; the
        rows outside every sequence are left as they were)."""
        n, seqs, at = q.shape[0], cu_seqlens.numel() - 1, self.workspace.device
        if out is None:
            out = torch.empty((n, self.num_q_heads, self.head_dim), dtype=q.dtype, device=q.device)
        if n > self.max_tokens or not 0 <= seqs <= self.max_seqs:
            raise ValueError(f"{n} tokens in {seqs} sequences, the workspace holds {self.max_tokens} in {self.max_seqs}")
        for name, x, h in (("q", q, self.num_q_heads), ("k", k, self.num_kv_heads), ("v", v, self.num_kv_heads),
                           ("out", out, self.num_q_heads)):
            if x.shape != (n, h, self.head_dim) or x.dtype != TORCH_DT[self.dtype] or x.device != at:
                raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, expected "
                                 f"{(n, h, self.head_dim)} {TORCH_DT[self.dtype]} on {at}")
            if x.stride(2) != 1 or (h > 1 and x.stride(1) != self.head_dim):
                raise ValueError(f"{name}: each token's heads must be contiguous")
        if cu_seqlens.dtype != torch.int32 or cu_seqlens.device != at or not cu_seqlens.is_contiguous():
            raise ValueError("cu_seqlens: contiguous int32 on the workspace's device expected")
        row = lambda x: x.stride(0) if n > 1 else x.shape[1] * x.shape[2]  # noqa: E731
        a = B.GbPromptArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), cu_seqlens.data_ptr(),
                           self.workspace.data_ptr(), self.workspace.numel(), row(q), row(k), row(v), row(out), seqs, n,
                           self.num_q_heads, self.num_kv_heads, self.head_dim, _DT[self.dtype], scale)
        B.gb_prompt_attention(a, stream)
        return out

    def status(self, stream=None) -> int:
        return B.gb_prompt_status(self.workspace, stream)
