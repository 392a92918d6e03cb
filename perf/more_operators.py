"""Operators measured here: what one generated token of a beam search takes besides the model's products, over a
pool whose keys and values are held in 8 bits.

Three kinds of case:

* ``step``     ``BeamPool.decode_attention`` with a ``Rotation`` on an 8-bit pool, every layer: the step's queries and
               keys are rotated to their positions, the new rows join the cache in 8 bits, every trace attends to its
               whole context.  ``BeamPool.truncate`` then takes the token back, so that a pass can be made again.
* ``thought``  ``BeamPool.append_kv`` with a ``Rotation``: a chunk of tokens joins every trace's cache at once (8-bit,
               bf16 and fp32 pools); ``BeamPool.read_kv`` returns what the cache then holds; ``truncate`` takes it back.
* ``sample``   ``TokenSampler``: the next token of every trace from its logits and a given random number, with
               temperature, top-k, min-p and top-p, and the token's log-probability.

The caches are beam trees: ``beams`` traces over a shared prompt, and after every ``interval`` tokens half of
them give way to branches of others, which share their parent's pages.  Shapes (lengths, trees, forks) come from
the case, values from the seed.

An 8-bit cache holds e4m3 values and, for each block of 16 tokens (by position) of a head, a power of two that they
are multiplied by: the smallest 2^e, e in [-60, 60], with all of the block's rows within 448 2^e.  A row that does not
fit raises its block's e, and the rows before it are rounded again.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.bfloat16}   # of the rows that a caller gives
BLOCK, E_LEAST, E_MOST, TOP = 16, -60, 60, 448.0
NO = -1e30           # below every score; exp of it is 0
BASE = 1e6           # of the rotation's frequencies


# --------------------------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------------------------

def _tree(kind, name, **kw):
    c = {"name": name, "kind": kind, "dtype": "fp8", "slots": 64, "beams": 64, "prompt": 512, "context": 4000,
         "interval": 512, "tokens": 1, "layers": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 16,
         "rotary": 128, "interleaved": False, "shape": 1}
    c.update(kw)
    return c


def _sample(name, **kw):
    c = {"name": name, "kind": "sample", "dtype": "bf16", "rows": 64, "vocab": 128000, "pad": 0, "top_k": 0, "top_p": 1.0,
         "min_p": 0.0, "temperature": 0.6, "mixed": False, "banned": 0.0, "sharp": 2.5, "shape": 1}
    c.update(kw)
    return c


def listed():
    return [
        # The smallest search's traces: latency only.
        _tree("step", "step_8", slots=8, beams=8, prompt=64, context=250, interval=96, q_heads=4, kv_heads=2),
        # A small interactive search over a few layers, pages of 64 tokens, slots without a trace.
        _tree("step", "step_13", slots=16, beams=13, prompt=333, context=700, interval=150, layers=4, page=64),
        # One long trace: few rows over a long cache; half of each head is rotated.
        _tree("step", "step_single_20k", slots=1, beams=1, prompt=20000, context=20000, interval=0, rotary=64),
        # The ordinary search: 64 traces at 4K that share most of their contexts.
        _tree("step", "step_64x4k", layers=2),
        # Many traces at 8K, eight query heads per KV head, slots that hold no trace.
        _tree("step", "step_198x8k", slots=210, beams=198, context=8000, kv_heads=4),
        # Traces that share nothing: the cache is read at the memory's rate.
        _tree("step", "step_unshared_64x16k", prompt=1, context=16384, interval=0),
        # A short thought of the smallest search, fp32.
        _tree("thought", "thought_8_f32", dtype="f32", slots=8, beams=8, prompt=64, context=150, interval=96, tokens=24,
              q_heads=4, kv_heads=2, head_dim=64, rotary=64),
        # Thoughts of an ordinary search over a few layers, bf16, interleaved pairs.
        _tree("thought", "thought_64_bf16", dtype="bf16", prompt=300, context=300, tokens=33, layers=4, interleaved=True),
        # A long thought of every trace of a large search at once: the copying counts.
        _tree("thought", "thought_256_fp8", slots=256, beams=256, prompt=200, context=405, interval=205, tokens=199),
        # A few traces' next tokens, a small vocabulary: latency only.
        _sample("sample_8_32k", rows=8, vocab=32000, top_k=20, top_p=0.95),
        # The ordinary search's next tokens by nucleus alone, fp32 logits of a padded projection.
        _sample("sample_64_nucleus", dtype="f32", vocab=151000, pad=64, top_p=0.95),
        # Many traces, every row with parameters of its own (greedy ones and plain ones among them), banned tokens.
        _sample("sample_512_mixed", rows=512, mixed=True, banned=0.01, temperature=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "thought", "sample", "sample"])
    if kind == "sample":
        c = _sample("", dtype=rng.choice(["bf16", "f32"]), rows=_log(rng, 1, 512), vocab=_log(rng, 100, 160000),
                    pad=rng.choice([0, 0, rng.randint(1, 200)]), top_k=rng.choice([0, 0, _log(rng, 1, 200)]),
                    top_p=rng.choice([1.0, round(rng.uniform(0.5, 0.999), 3)]),
                    min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 3)]), temperature=round(rng.uniform(0.1, 1.5), 2),
                    mixed=rng.random() < 0.3, banned=rng.choice([0.0, 0.02, 0.5]), sharp=round(rng.uniform(0.3, 5.0), 1),
                    shape=rng.randrange(1, 1 << 30))
        while c["rows"] * c["vocab"] > 512 * 128000:
            c["rows"] = max(1, c["rows"] // 2)
        return c
    dtype = "fp8" if kind == "step" else rng.choice(["fp8", "fp8", "bf16", "f32"])
    d = 64 if dtype == "f32" else 128
    kvh = rng.choice([1, 2, 4, 8])
    c = _tree(kind, "", dtype=dtype, beams=_log(rng, 1, 200), prompt=_log(rng, 1, 4096), layers=rng.choice([1, 2, 4]),
              page=rng.choice([16, 32, 64]), kv_heads=kvh, q_heads=kvh * rng.choice([2, 4, 8]), head_dim=d,
              rotary=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.random() < 0.3, shape=rng.randrange(1, 1 << 30))
    c["slots"] = c["beams"] + rng.choice([0, 0, _log(rng, 1, 64)])
    c["interval"] = _log(rng, 64, 1024)
    c["context"] = c["prompt"] + rng.choice([0, c["interval"], 3 * c["interval"] + rng.randint(1, 63), _log(rng, 1, 6000)])
    if kind == "thought":
        c["context"] = min(c["context"], c["prompt"] + 2 * c["interval"])
        c["tokens"] = _log(rng, 1, 400)
    while c["beams"] * c["layers"] * kvh * (c["context"] * 400 + c["tokens"] * 6000) > 2.4e9:
        c["layers"] = 1
        c["beams"], c["tokens"] = max(1, c["beams"] * 3 // 4), max(1, c["tokens"] * 3 // 4)
    c["slots"] = max(c["beams"], min(c["slots"], c["beams"] + 64))
    return c


def _grow(case):
    """The beams' contexts: (rows of the token store by beam and position, rows used, rounds), a round being
    (first position, tokens, first row of the store, parents of the fork that follows or None)."""
    rng = np.random.RandomState(case["shape"])
    beams, prompt, context, step = case["beams"], case["prompt"], case["context"], case["interval"]
    rows = np.zeros((beams, context), np.int64)
    rows[:, :prompt] = np.arange(prompt)
    at, used, rounds = prompt, prompt, []
    while at < context:
        n = min(step, context - at) if step else context - at
        first, used = used, used + beams * n
        rows[:, at:at + n] = first + np.arange(beams * n).reshape(beams, n)
        parents = None
        if at + n < context and beams > 1:
            order = rng.permutation(beams)
            parents = np.arange(beams)
            parents[order[:beams // 2]] = order[beams // 2:][np.arange(beams // 2)]
            rows[:, :at + n] = rows[parents, :at + n]
        rounds.append((at, n, first, parents))
        at += n
    return rows, used, rounds


# --------------------------------------------------------------------------------------------
# What a program has before the call
# --------------------------------------------------------------------------------------------

def _cache_rows(g, layers, n, heads, d, dtype):
    """Keys or values: N(0, 1), louder in some channels of a head, and louder in some tokens."""
    out = torch.empty(layers, n, heads, d, dtype=dtype, device="cuda")
    for layer in range(layers):
        loud = torch.randn(heads, d, generator=g, device="cuda").mul_(0.5).exp_()
        for i in range(0, n, 1 << 16):
            x = out[layer, i:i + (1 << 16)]
            token = torch.randn(x.shape[0], 1, 1, generator=g, device="cuda").mul_(0.3).exp_()
            x.copy_(torch.randn(x.shape, generator=g, device="cuda").mul_(loud).mul_(token))
    return out


def _two(e):
    """2^e in 32 bits."""
    return ((e + 127) << 23).view(torch.float32)


def _held(x, e):
    """The values that e4m3 holds of x at the scale 2^e."""
    return (x / _two(e)).to(torch.float8_e4m3fn).float() * _two(e)


def _extend(values, e, x, at):
    """Rows x [beams][n][heads][d] join a cache of 8 bits at position `at`: (the values of every block that they reach,
    from the first block's start on, and those blocks' exponents).  values [beams][at ..][heads][d] and
    e [beams][blocks][heads] are the cache before."""
    b, n, h, d = x.shape
    lo, hi = at // BLOCK * BLOCK, -(-(at + n) // BLOCK) * BLOCK
    new = torch.zeros(b, hi - lo, h, d, device=x.device)
    new[:, at - lo:at - lo + n] = x.float()
    m, ex = torch.frexp(new.abs().unflatten(1, (-1, BLOCK)).amax((2, 4)))
    need = torch.where(m > 0, ex - 9 + (m > TOP / 512).int(), torch.full_like(ex, E_LEAST)).clamp_(E_LEAST, E_MOST)
    if at > lo:
        new[:, :at - lo] = values[:, lo:at].float()
        need[:, 0] = torch.maximum(need[:, 0], e[:, lo // BLOCK])
    return _held(new.unflatten(1, (-1, BLOCK)), need[:, :, None, :, None]).flatten(1, 2), need


def _fill(case, rounds, store, layer):
    """One layer's 8-bit cache, [beams][context] values (e4m3 codes) and scales, grown as the pool grows."""
    beams, context = case["beams"], case["context"]
    blocks = -(-context // BLOCK)
    h, d = store.shape[2:]
    values = torch.zeros(beams, blocks * BLOCK, h, d, device="cuda")
    e = torch.full((beams, blocks, h), E_LEAST, dtype=torch.int32, device="cuda")
    p = case["prompt"]
    v, x = _extend(values[:1], e[:1], store[layer, None, :p], 0)
    values[:, :v.shape[1]], e[:, :x.shape[1]] = v, x
    for at, n, first, parents in rounds:
        for i in range(0, beams, 32):   # (in parts: the rows of many long traces in 32 bits)
            rows = store[layer, first:first + beams * n].unflatten(0, (beams, n))[i:i + 32]
            v, x = _extend(values[i:i + 32], e[i:i + 32], rows, at)
            lo = at // BLOCK * BLOCK
            values[i:i + 32, lo:lo + v.shape[1]], e[i:i + 32, lo // BLOCK:lo // BLOCK + x.shape[1]] = v, x
        if parents is not None:
            to = torch.from_numpy(parents).cuda()
            moved = (to != torch.arange(beams, device="cuda")).nonzero()[:, 0]
            values[moved, :at + n], e[moved] = values[to[moved], :at + n], e[to[moved]]
    return values.unflatten(1, (-1, BLOCK)).div_(_two(e)[:, :, None, :, None]).flatten(1, 2).to(torch.float8_e4m3fn), e


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "sample":
        return _prepare_sample(case, s, g)
    hq, hkv, d, dt = case["q_heads"], case["kv_heads"], case["head_dim"], DT[case["dtype"]]
    rows, used, rounds = _grow(case)
    slots, beams, layers, t = case["slots"], case["beams"], case["layers"], case["tokens"]
    store = {x: _cache_rows(g, layers, used, hkv, d, dt) for x in ("k", "v")}
    s["q"] = torch.randn(layers, slots, hq, d, generator=g, device="cuda").to(dt)
    for x in ("k", "v"):
        s["new_" + x] = _cache_rows(g, layers, t * slots, hkv, d, dt).unflatten(1, (t, slots))
    s["scale"] = 1 / math.sqrt(d)
    s["first"] = torch.full((slots,), case["context"], dtype=torch.int32, device="cuda")
    s["out"] = torch.zeros(layers, slots, hq, d, device="cuda")
    if not own:
        if case["dtype"] == "fp8":
            s["cache"] = [{x: _fill(case, rounds, store[x], i) for x in ("k", "v")} for i in range(layers)]
        return s
    from paper_2608_08020_gb300.pool import BeamPool
    from paper_2608_08020_gb300.rotation import Rotation
    width = -(-(case["context"] + t) // case["page"]) + 1
    pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=case["page"],
                    kv_dtype=case["dtype"], num_pages=used // case["page"] + (2 * len(rounds) + t // case["page"] + 8) * beams + 64,
                    max_beams=slots, max_pages_per_beam=width)
    p = case["prompt"]
    pool.seed(beams, p, store["k"][:, :p].contiguous(), store["v"][:, :p].contiguous())
    for _, n, first, parents in rounds:   # the store holds a round's rows beam by beam
        for layer in range(layers):
            x = torch.zeros(2, n, slots, hkv, d, dtype=dt, device="cuda")
            for kv in (0, 1):
                x[kv, :, :beams] = store["kv"[kv]][layer, first:first + beams * n].unflatten(0, (beams, n)).transpose(0, 1)
            pool.append_kv(layer, n, x[0], x[1])
        if parents is not None:
            pf = np.full(slots, -1, np.int32)
            pf[:beams] = parents
            pool.fork_slots(torch.from_numpy(pf).cuda())
    assert pool.status() == 0
    s["pool"] = pool
    s["rotation"] = Rotation(d, max_positions=case["context"] + t, base=BASE, rotary_dim=case["rotary"],
                             interleaved=case["interleaved"])
    return s


def _prepare_sample(case, s, g):
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn(rows, vocab + case["pad"], generator=g, device="cuda").mul_(case["sharp"])
    # A few likely tokens in every row, more or less ahead of the rest.
    ahead = torch.randn(rows, 1, generator=g, device="cuda").mul_(0.5).exp_().mul_(case["sharp"])
    likely = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
    x.scatter_add_(1, likely, ahead * torch.empty(rows, 24, device="cuda").exponential_(generator=g))
    if case["banned"]:
        x.masked_fill_(torch.rand(x.shape, generator=g, device="cuda") < case["banned"], -math.inf)
    s["logits"] = x.to(DT[case["dtype"]])[:, :vocab]
    s["u"] = torch.rand(rows, generator=g, device="cuda")
    # Each row's parameters: the case's, or drawn from what requests ask for (0 is greedy, off, off).
    rng = np.random.RandomState(case["shape"])
    some = (lambda *a: rng.choice(a, rows)) if case["mixed"] else None
    given = {"temperature": (torch.float32, (0.0, 0.3, 0.6, 1.0, 1.2)), "top_k": (torch.int32, (0, 0, 1, 20, 50)),
             "top_p": (torch.float32, (1.0, 0.8, 0.9, 0.95)), "min_p": (torch.float32, (0.0, 0.0, 0.05, 0.1))}
    for name, (dt, values) in given.items():
        s[name] = torch.tensor(some(*values) if some else [case[name]] * rows, dtype=dt, device="cuda")
    if own:
        from paper_2608_08020_gb300.sampling import TokenSampler
        s["op"] = TokenSampler(max_rows=rows, vocab=vocab)
    return s


# --------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if kind == "sample":
        if own:
            token, logprob = s["op"](s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                     min_p=s["min_p"])
            return {"token": token, "logprob": logprob}
        return _plain_sample(s)
    if not own:
        return _plain_step(s) if kind == "step" else _plain_thought(s)
    pool, layers = s["pool"], s["case"]["layers"]
    if kind == "step":
        for i in range(layers):
            pool.decode_attention(i, s["q"][i], s["new_k"][i, 0], s["new_v"][i, 0], s["scale"], s["out"][i], rotation=s["rotation"])
        out = s["out"]
    else:
        n = s["case"]["tokens"]
        for i in range(layers):
            pool.append_kv(i, n, s["new_k"][i], s["new_v"][i], rotation=s["rotation"])
        out = [pool.read_kv(i, s["first"], n) for i in range(layers)]
    pool.truncate(s["first"])
    return out


def _rotate(x, at, case):
    """x [tokens][...][d], token i at position at + i, rotated; in 64 bits, as what follows rounds it to 16 or 8."""
    r = case["rotary"]
    f = BASE ** (-torch.arange(0, r, 2, dtype=torch.float64, device=x.device) / r)
    angle = torch.arange(at, at + x.shape[0], dtype=torch.float64, device=x.device)[:, None] * f
    c, n = (t.reshape(x.shape[0], *[1] * (x.dim() - 2), -1) for t in (angle.cos(), angle.sin()))
    x = x.double()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * c - b * n, b * c + a * n
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _tail(codes, e, at):
    """The cache's rows of the block that position `at` lies in, as values, and its exponents."""
    lo = at // BLOCK * BLOCK
    e = e[:, lo // BLOCK:]
    return codes[:, lo:at].float() * _two(e[:, :1, :, None]) if at > lo else None, e


def _plain_step(s):
    """Every trace's whole cache out of its 8 bits, the blocks that the new token reaches replaced, all scores at once."""
    case = s["case"]
    beams, at, hkv, hq = case["beams"], case["context"], case["kv_heads"], case["q_heads"]
    g, lo = hq // hkv, at // BLOCK * BLOCK
    out = torch.zeros(case["layers"], case["slots"], hq, case["head_dim"], device="cuda")
    for i in range(case["layers"]):
        q = _rotate(s["q"][i, None, :beams], at, case)[0].to(s["q"].dtype).float()
        kv = []
        for x in ("k", "v"):
            new = s["new_" + x][i, :, :beams]
            new = (_rotate(new, at, case) if x == "k" else new).transpose(0, 1)
            codes, e = s["cache"][i][x]
            held = codes[:, :lo].float().unflatten(1, (-1, BLOCK)).mul_(_two(e[:, :lo // BLOCK])[:, :, None, :, None]).flatten(1, 2)
            tail = _extend(*_tail(codes, e, at), new, at - lo)[0]
            kv.append(torch.cat([held, tail[:, :at + 1 - lo]], 1).permute(0, 2, 3, 1))    # [beams][hkv][d][tokens]
            del held
        x = torch.matmul(q.unflatten(1, (hkv, g)), kv[0]).mul_(s["scale"])
        x.sub_(x.amax(-1, keepdim=True)).exp_()
        x.div_(x.sum(-1, keepdim=True))
        out[i, :beams] = torch.matmul(x, kv[1].transpose(2, 3)).flatten(1, 2)
    return out


def _plain_thought(s):
    """The appended tokens as the cache holds them, by layer: (keys, values) [tokens][slots][heads][d]."""
    case = s["case"]
    beams, at, n = case["beams"], case["context"], case["tokens"]
    out = []
    for i in range(case["layers"]):
        kv = []
        for x in ("k", "v"):
            new = s["new_" + x][i, :, :beams]
            new = (_rotate(new, at, case) if x == "k" else new)
            if case["dtype"] == "fp8":
                codes, e = s["cache"][i][x]
                off = at % BLOCK
                new = _extend(*_tail(codes, e, at), new.transpose(0, 1), off)[0][:, off:off + n].transpose(0, 1)
            held = torch.zeros_like(s["new_" + x][i])
            held[:, :beams] = new.to(held.dtype)
            kv.append(held)
        out.append(tuple(kv))
    return out


def _plain_sample(s):
    """Every row sorted, in 64 bits: sums over a whole vocabulary are compared with a random number."""
    x = s["logits"].double()
    t, k, p, m = (s[n].double()[:, None] for n in ("temperature", "top_k", "top_p", "min_p"))
    v, at = x.sort(dim=-1, descending=True, stable=True)
    rank = torch.arange(x.shape[1], device=x.device)
    y = (v - v[:, :1]).div_(torch.where(t > 0, t, 1.0))
    keep = ((k <= 0) | (rank < k)) & (y >= m.log()) & ((t > 0) | (rank < 1))
    w = y.exp_().mul_(keep)
    c = w.cumsum(-1)
    w.mul_((p >= 1) | (c - w < p * c[:, -1:]))
    w = torch.zeros_like(w).scatter_(1, at, w)
    c = w.cumsum(-1)
    token = (c <= s["u"].double()[:, None] * c[:, -1:]).sum(-1, keepdim=True)
    return {"token": token[:, 0].int(), "logprob": (w.gather(1, token) / c[:, -1:]).log()[:, 0].float()}


# --------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "sample":
        n = float(case["rows"] * case["vocab"])
        # The logits read once; of each value a comparison, an exponential and a sum.
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + case["rows"] * 28, "flops": 4 * n}
    hq, hkv, d, beams, t = case["q_heads"], case["kv_heads"], case["head_dim"], case["beams"], case["tokens"]
    es = 4 if case["dtype"] == "f32" else 2
    held = d + 1 / BLOCK if case["dtype"] == "fp8" else d * es       # bytes of a cached row
    new = beams * t * hkv * 2 * (d * es + held)                     # read, and written to the cache
    if case["kind"] == "thought":
        back = beams * t * hkv * 2 * held + case["slots"] * t * hkv * 2 * d * es
        return {"bytes": case["layers"] * (new + back), "flops": case["layers"] * beams * t * hkv * 3 * case["rotary"]}
    rows, _, _ = _grow(case)
    seen = float(np.unique(rows).size)                               # tokens that some trace still holds, each read once
    b = seen * hkv * 2 * held + new + beams * hq * d * 2 + case["slots"] * hq * d * 4
    return {"bytes": case["layers"] * b, "flops": case["layers"] * beams * (case["context"] + 1.0) * hq * 4 * d}


# --------------------------------------------------------------------------------------------
# The definition, in 64 bits
# --------------------------------------------------------------------------------------------

def _turned(x, at, case):
    """One token's heads x [heads][d] in 64 bits at position `at`: pairs as complex numbers, turned."""
    r = case["rotary"]
    x = x.double()
    i = torch.arange(r // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
    z = torch.complex(x[:, a], x[:, b]) * torch.polar(torch.ones_like(i, dtype=torch.float64), at * BASE ** (-2 * i.double() / r))
    y = x.clone()
    y[:, a], y[:, b] = z.real, z.imag
    return y


def _pow2(e):
    """2^e in 64 bits, exactly (values that lie between two others are rounded by it)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round8(x, e):
    """x [...][rows][d] in 64 bits to the nearest value of 4 significant bits (3 below 2^-6) times 2^e[...], ties to even."""
    x = x / _pow2(e)[..., None, None]
    step = _pow2((torch.frexp(x)[1] - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step * _pow2(e)[..., None, None]


def _exponent(x):
    """The least e with |x| <= 448 2^e, of each [rows][d]."""
    most = x.abs().amax((-2, -1))
    e = torch.ceil(torch.log2(most / TOP)).clamp(E_LEAST, E_MOST).int()
    e = e + (most > TOP * _pow2(e)).int() - (most <= TOP * _pow2(e - 1)).int()      # (where log2 was off)
    return torch.where(most > 0, e, E_LEAST).clamp(E_LEAST, E_MOST)


def _exact_blocks(case, s, layer, x, b):
    """What slot b's cache holds from its last block's start on once the new tokens are in, [rows][heads][d], from the
    codes and scales that it held before."""
    at, n = case["context"], case["tokens"]
    codes, e = s["cache"][layer][x]
    new = torch.stack([_turned(y, at + j, case) if x == "k" else y.double() for j, y in enumerate(s["new_" + x][layer, :, b])])
    lo = at // BLOCK * BLOCK
    done = []
    for first in range(lo, at + n, BLOCK):
        rows = new[max(first - at, 0):first + BLOCK - at].transpose(0, 1)          # [heads][rows][d]
        to = _exponent(rows)
        if first < at:
            was = e[b, first // BLOCK]
            to = torch.maximum(to, was)
            rows = torch.cat([codes[b, first:at].double().transpose(0, 1) * _pow2(was)[:, None, None], rows], 1)
        done.append(_round8(rows, to).transpose(0, 1))
    return torch.cat(done)


def exact(case, seed):
    if work(case)["flops"] > 2e11 or case["kind"] == "thought" and case["beams"] * case["tokens"] * case["layers"] > 12000:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "sample":
        return {"token": None, "logprob": torch.stack([_exact_row(s, r) for r in range(case["rows"])])}
    hq, hkv, at, n = case["q_heads"], case["kv_heads"], case["context"], case["tokens"]
    lo = at // BLOCK * BLOCK
    if case["kind"] == "thought":
        out = []
        for i in range(case["layers"]):
            kv = []
            for x in ("k", "v"):
                y = torch.zeros(s["new_" + x][i].shape, dtype=torch.float64, device="cuda")
                for b in range(case["beams"]):
                    if case["dtype"] == "fp8":
                        y[:, b] = _exact_blocks(case, s, i, x, b)[at - lo:]
                    else:
                        for j in range(n):
                            z = s["new_" + x][i, j, b]
                            y[j, b] = _turned(z, at + j, case) if x == "k" else z.double()
                kv.append(y)
            out.append(tuple(kv))
        return out
    out = torch.zeros(case["layers"], case["slots"], hq, case["head_dim"], dtype=torch.float64, device="cuda")
    for i in range(case["layers"]):
        for b in range(case["beams"]):
            kv = []
            for x in ("k", "v"):
                codes, e = s["cache"][i][x]
                blocks = codes[b, :lo].double().unflatten(0, (-1, BLOCK)) * _pow2(e[b, :lo // BLOCK])[:, None, :, None]
                kv.append(torch.cat([blocks.flatten(0, 1), _exact_blocks(case, s, i, x, b)]).transpose(0, 1))
            # The query that the scores are of is a bf16 one, as a model's rotated queries are.
            q = _turned(s["q"][i, b], at, case).to(s["q"].dtype).double().unflatten(0, (hkv, hq // hkv))
            p = torch.softmax(q @ kv[0].transpose(1, 2) * s["scale"], -1)
            out[i, b] = (p @ kv[1]).flatten(0, 1)
    return out


def _exact_row(s, r):
    """One row's log-probability of its token: kept tokens walked from the likeliest down, then the draw by index."""
    x, t, k, p, m = s["logits"][r].double(), *(s[n][r].item() for n in ("temperature", "top_k", "top_p", "min_p"))
    if not t > 0:
        return torch.zeros((), dtype=torch.float64, device="cuda")
    w = torch.exp((x - x.max()) / t)
    if m > 0:
        w[(x - x.max()) / t < math.log(m)] = 0
    order = torch.argsort(x, descending=True, stable=True)
    if k > 0:
        w[order[k:]] = 0
    if p < 1:
        before = torch.cumsum(w[order], 0) - w[order]
        w[order[before >= p * w.sum()]] = 0
    c = torch.cumsum(w, 0)
    i = int(torch.searchsorted(c, s["u"][r].double() * c[-1], right=True))
    return torch.log(w[i] / c[-1])
