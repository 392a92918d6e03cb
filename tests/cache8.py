"""A beam pool of 8 bits, as it is defined, in 64 bits on the CPU: each slot's rows as the cache holds them.  Plain lists
of blocks, no pages (the page accounting has oracles of its own)."""
import torch

BLOCK, LEAST, MOST = 16, -60, 60


def nearest_e4m3(x):
    """The nearest value of 4 significant bits (3 fewer places below 2^-6), ties to even; 448 past the end, NaN stays."""
    mant, ex = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (ex - 4).clamp(min=-9))
    y = (torch.round(x / step) * step).clamp(-448.0, 448.0)
    return torch.where(torch.isnan(x), x, y)


def least_exponent(x):
    """The least e in range with every finite value of x within 448 2^e."""
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).max().item()
    e = LEAST
    while e < MOST and top > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache8:
    def __init__(self, layers, slots, heads, d):
        self.shape = (layers, heads, d)
        self.kv = [[None] * layers for _ in range(slots)]     # [slot][layer]: (rows [2][T][heads][d], exps [2][blocks][heads])

    def length(self, b):
        return 0 if self.kv[b][0] is None else self.kv[b][0][0].shape[1]

    def append(self, b, layer, k, v):
        """k, v [n][heads][d] float64: rows at the slot's end."""
        _, heads, d = self.shape
        rows, exps = self.kv[b][layer] if self.kv[b][layer] is not None else (torch.zeros(2, 0, heads, d, dtype=torch.float64),
                                                                              torch.zeros(2, 0, heads, dtype=torch.int64))
        at, n = rows.shape[1], k.shape[0]
        new = torch.stack([k, v])
        new = torch.where(torch.isfinite(new), new, torch.full_like(new, float("nan")))
        rows = torch.cat([rows, new], 1)
        blocks = -(-(at + n) // BLOCK)
        exps = torch.cat([exps, torch.full((2, blocks - exps.shape[1], heads), LEAST, dtype=torch.int64)], 1)
        for j in range(at // BLOCK, blocks):
            lo, hi = max(at, j * BLOCK), min(at + n, (j + 1) * BLOCK)
            for kv in range(2):
                for h in range(heads):
                    need = least_exponent(rows[kv, lo:hi, h])
                    was = int(exps[kv, j, h]) if lo > j * BLOCK else LEAST
                    e = max(need, was)
                    f = 2.0 ** e
                    rows[kv, lo:hi, h] = nearest_e4m3(rows[kv, lo:hi, h] / f) * f
                    if e != was and lo > j * BLOCK:
                        rows[kv, j * BLOCK:lo, h] = nearest_e4m3(rows[kv, j * BLOCK:lo, h] / f) * f
                    exps[kv, j, h] = e
        self.kv[b][layer] = (rows, exps)

    def fork(self, parent_of):
        self.kv = [list(self.kv[p]) if p >= 0 else self.kv[b] for b, p in enumerate(parent_of)]

    def truncate(self, b, n):
        self.kv[b] = [(r[:, :n].clone(), e[:, :-(-n // BLOCK)].clone()) for r, e in self.kv[b]]

    def release(self, b):
        self.kv[b] = [None] * len(self.kv[b])

    def read(self, layer, first, n):
        """[2][n][slots][heads][d] of tokens first[b] ..; zeros where a slot has none."""
        _, heads, d = self.shape
        out = torch.zeros(2, n, len(self.kv), heads, d, dtype=torch.float64)
        for b in range(len(self.kv)):
            for i in range(n):
                t = first[b] + i
                if 0 <= t < self.length(b):
                    out[:, i, b] = self.kv[b][layer][0][:, t]
        return out


def rotated(x, pos, rotary, base, interleaved=False, amplitude=1.0):
    """x [..][d] float64 at position pos."""
    i = torch.arange(rotary // 2)
    angle = pos * base ** (-2.0 * i.double() / rotary)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    y = x.clone()
    y[..., a] = (x[..., a] * angle.cos() - x[..., b] * angle.sin()) * amplitude
    y[..., b] = (x[..., b] * angle.cos() + x[..., a] * angle.sin()) * amplitude
    return y


def attention(q, held, scale):
    """q [Hq][D] over what a slot's cache holds, and what its rounding is measured by: (out, sum p |v|, the largest
    sum |q_i k_i| scale, the largest p 2^e of V), by head."""
    rows, exps = held
    g = q.shape[0] // rows.shape[2]
    k, v = (rows[i].repeat_interleave(g, 1).transpose(0, 1) for i in (0, 1))      # [Hq][T][D]
    p = ((k @ q[:, :, None])[..., 0] * scale).softmax(-1)
    size = (k.abs() @ q.abs()[:, :, None])[..., 0].amax(-1) * scale
    f = torch.ldexp(torch.ones(exps.shape[1:], dtype=torch.float64), exps[1])     # [blocks][heads]
    f = f.repeat_interleave(BLOCK, 0)[:rows.shape[1]].repeat_interleave(g, 1).T
    return (p[:, None] @ v)[:, 0], (p[:, None] @ v.abs())[:, 0], size, (p * f).amax(-1)
