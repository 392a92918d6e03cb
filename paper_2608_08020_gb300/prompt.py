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
        self.max_tokens, self.max_seqs = max_tokens, max_seqs
        n = B.gb_prompt_workspace_bytes(max_tokens, max_seqs, num_q_heads, num_kv_heads, head_dim, _DT[dtype])
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=torch.device(device))   # status: GB_OK
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.workspace.device).synchronize()                # calls may be on any stream
        self.device, self.torch_dtype = self.workspace.device, TORCH_DT[dtype]
        self._index = self.device.index
        # The call's arguments, but for what changes from call to call.
        self._args = B.GbPromptArgs(workspace=self.workspace.data_ptr(), workspace_bytes=n, num_q_heads=num_q_heads,
                                    num_kv_heads=num_kv_heads, head_dim=head_dim, dtype=_DT[dtype])

    def __call__(self, q, k, v, cu_seqlens, scale: float, out=None, stream=None):
        """q [tokens][q heads][head_dim], k and v [tokens][kv heads][head_dim] (each token's heads contiguous, tokens
        at any stride), cu_seqlens int32 [seqs + 1]; returns out [tokens][q heads][head_dim] (new unless given; the
        rows outside every sequence are left as they were).  A new out belongs to `stream`, which then has to be a
        torch.cuda.Stream or None."""
        n, seqs = q.shape[0], cu_seqlens.numel() - 1
        if out is None:
            out = torch.empty_like(q) if stream is None else B.new_on(stream, lambda: torch.empty_like(q))
        if n > self.max_tokens or not 0 <= seqs <= self.max_seqs:
            raise ValueError(f"{n} tokens in {seqs} sequences, the workspace holds {self.max_tokens} in {self.max_seqs}")
        a = self._args
        a.q, a.q_stride = self._rows("q", q, n, self.num_q_heads)
        a.k, a.k_stride = self._rows("k", k, n, self.num_kv_heads)
        a.v, a.v_stride = self._rows("v", v, n, self.num_kv_heads)
        a.out, a.out_stride = self._rows("out", out, n, self.num_q_heads)
        if cu_seqlens.dtype is not torch.int32 or cu_seqlens.get_device() != self._index or not cu_seqlens.is_contiguous():
            raise ValueError("cu_seqlens: contiguous int32 on the workspace's device expected")
        a.cu_seqlens, a.num_seqs, a.num_tokens, a.scale = cu_seqlens.data_ptr(), seqs, n, scale
        B.gb_prompt_attention(a, stream, self._index)
        return out

    def _rows(self, name, x, n, heads):
        """Address and token stride of a tensor of rows."""
        d = self.head_dim
        if x.shape != (n, heads, d) or x.dtype is not self.torch_dtype or x.get_device() != self._index:
            raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, expected {(n, heads, d)} {self.torch_dtype} "
                             f"on {self.device}")
        token, head, one = x.stride()
        if one != 1 or (heads > 1 and head != d):
            raise ValueError(f"{name}: each token's heads must be contiguous")
        return x.data_ptr(), token if n > 1 else heads * d

    def status(self, stream=None) -> int:
        """Device status of the last call (synchronises)."""
        return B.gb_prompt_status(self.workspace, stream)
