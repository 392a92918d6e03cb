"""``Rotation``: rotary position embedding for the rows on their way into a ``BeamPool``'s cache.

``BeamPool.append_kv`` and ``BeamPool.decode_attention`` take one: keys (and a decode step's queries) are then given as
the projection leaves them, and the library turns them to the positions that they are appended at, which only the pool
on the device knows.  The object is the table of angles; it belongs to no pool and may serve many.  It may be dropped while
calls that use it are still to run, but for those on a raw stream handle and those in a captured graph, which reads the table
at each replay: for these the caller keeps it.
"""
from __future__ import annotations

import torch

from paper_2608_08020_gb300 import binding as B


class Rotation:
    def __init__(self, head_dim: int, *, max_positions: int, base: float = 10000.0, rotary_dim: int | None = None,
                 interleaved: bool = False, frequencies=None, amplitude: float = 1.0, device: str | torch.device = "cuda"):
        """Pairs (i, i + rotary_dim / 2) of each head's first rotary_dim values (all of them unless given), or (2i, 2i + 1)
        where `interleaved`, turn by frequencies[i] a position: base ** (-2 i / rotary_dim) unless given (float64, any scaling
        of long contexts already in them).  `amplitude` multiplies what is turned."""
        r = head_dim if rotary_dim is None else rotary_dim
        if r % 16 or not 16 <= r <= head_dim:
            raise ValueError(f"rotary_dim {r}: a multiple of 16 up to head_dim ({head_dim}) expected")
        if not 1 <= max_positions < 1 << 31:
            raise ValueError(f"max_positions {max_positions}")
        self.device = torch.device(device)
        if frequencies is None:
            f = base ** (-torch.arange(0, r, 2, dtype=torch.float64, device=self.device) / r)
        else:
            f = torch.as_tensor(frequencies, dtype=torch.float64).to(self.device)
            if f.shape != (r // 2,):
                raise ValueError(f"frequencies: {r // 2} expected, got {tuple(f.shape)}")
        self.head_dim, self.rotary_dim, self.max_positions, self.interleaved = head_dim, r, max_positions, bool(interleaved)
        # (cos, its rounding error, sin, its rounding error): the angles of far positions need 64 bits, and results are
        # rounded to 16 or 8 bits once, which a table of 32 bits alone would move across ties.
        self.table = torch.empty(max_positions, 4, r // 2, dtype=torch.float32, device=self.device)
        for at in range(0, max_positions, 1 << 16):
            part = self.table[at:at + (1 << 16)]
            angle = torch.arange(at, at + part.shape[0], dtype=torch.float64, device=self.device)[:, None] * f
            for i, exact in enumerate((angle.cos() * amplitude, angle.sin() * amplitude)):
                part[:, 2 * i] = exact
                part[:, 2 * i + 1] = exact - part[:, 2 * i].double()
        self.device = self.table.device
        if self.device.type == "cuda" and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.device).synchronize()       # calls may be on any stream
        # Streams that the table's memory waits for before others get it: the one that it comes from, and each that used it.
        self._streams = {torch.cuda.current_stream(self.device).cuda_stream} if self.device.type == "cuda" else set()
        self.args = B.GbRotation(self.table.data_ptr(), max_positions, r, int(self.interleaved))

    def used_on(self, stream) -> int:
        """The handle of `stream` (as BeamPool's calls take it), on which a call is about to read the table."""
        handle = B.stream_handle(stream)
        if handle not in self._streams and not isinstance(stream, int):
            self.table.record_stream(torch.cuda.current_stream(self.device) if stream is None else stream)
            self._streams.add(handle)
        return handle
