"""``TokenSampler``: every trace's next token from its logits, with temperature, top-k, min-p and top-p.

The step between a model's last product and its next ``BeamPool.decode_attention``.  The random numbers are the caller's, so
a search can be repeated.  Each call is one call of ``gb_sample``: one launch, no workspace.
"""
from __future__ import annotations

import torch

from paper_2608_08020_gb300 import binding as B

_DT = {torch.float32: B.GB_F32, torch.bfloat16: B.GB_BF16}
_OFF = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}
_TYPE = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}


class TokenSampler:
    def __init__(self, max_rows: int, vocab: int, *, device: str | torch.device = "cuda"):
        if max_rows < 1 or vocab < 1:
            raise ValueError(f"{max_rows} rows of {vocab} logits")
        self.max_rows, self.vocab = max_rows, vocab
        device = torch.device(device)
        self.device = device if device.index is not None else torch.device(device.type, torch.cuda.current_device())
        self._index = self.device.index

    def __call__(self, logits, u, *, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None, stream=None):
        """logits [rows][vocab] fp32 or bf16, each row contiguous, rows at any stride; u fp32 [rows] in [0, 1).  temperature, top_p,
        min_p (fp32) and top_k (int32): a number for all rows, a tensor [rows], or None (1, off, off, off); a temperature of 0 takes
        the likeliest token.  Returns (token int32 [rows], -1 where every logit is -infinity; logprob fp32 [rows], the natural
        logarithm of its share of the tokens kept), new ones unless given; they belong to `stream`, which then has to be a
        torch.cuda.Stream or None."""
        shape, stride, dtype = logits.shape, logits.stride(), _DT.get(logits.dtype)
        rows = shape[0]
        if len(shape) != 2 or rows > self.max_rows or shape[1] != self.vocab or dtype is None or logits.get_device() != self._index or \
                (stride[1] != 1 and self.vocab > 1) or (rows > 1 and stride[0] < self.vocab):
            raise ValueError(f"logits: {tuple(shape)} {logits.dtype} strides {stride} on {logits.device}, expected up to "
                             f"{self.max_rows} contiguous rows of {self.vocab} fp32 or bf16 values on {self.device}")
        if token is not None:
            self._row("token", token, rows, torch.int32)
        if logprob is not None:
            self._row("logprob", logprob, rows, torch.float32)
        if token is None or logprob is None:
            make = lambda: (torch.empty(rows, dtype=torch.int32, device=self.device) if token is None else token,  # noqa: E731
                            torch.empty(rows, dtype=torch.float32, device=self.device) if logprob is None else logprob)
            token, logprob = make() if stream is None else B.new_on(stream, make)
        row = {}                                   # a parameter's address, or None
        for name, x in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
            row[name] = self._row(name, x, rows, _TYPE[name]) if isinstance(x, torch.Tensor) else None
        if row["top_k"] is None and top_k is not None and not 0 < top_k < self.vocab:
            top_k = 0                              # off, also where the number has more than 32 bits
        number = lambda name, x: _OFF[name] if x is None or row[name] is not None else x  # noqa: E731
        # (In the order of the structure's fields: by name takes three times as long.)
        a = B.GbSampleArgs(logits.data_ptr(), stride[0] if rows > 1 else self.vocab, self._row("u", u, rows, torch.float32),
                           row["temperature"], row["top_k"], row["top_p"], row["min_p"], token.data_ptr(), logprob.data_ptr(), rows,
                           self.vocab, dtype, number("temperature", temperature), number("top_k", top_k), number("top_p", top_p),
                           number("min_p", min_p))
        B.gb_sample(a, stream, self._index)
        return token, logprob

    def _row(self, name, x, rows, dtype):
        if x.shape != (rows,) or x.dtype is not dtype or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, expected contiguous {(rows,)} {dtype} on {self.device}")
        return x.data_ptr()
