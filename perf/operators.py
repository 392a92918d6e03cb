"""Operators measured here: attention over prompts, attention for trees of drafted tokens over a beam pool's
cache, and the two calls that move a pool's beams along such a tree (accept a path, cut a beam short).

Three kinds of case:

* ``prompt``  ``PromptAttention``: causal attention over whole prompts, packed one after the other.
* ``draft``   ``DraftTrees.attention``: every beam's drafted tokens attend to the beam's cached context and to
              their own ancestors in the beam's tree; one pass is one call per layer.
* ``round``   ``DraftTrees.accept``, then ``attention`` of the next drafts over the grown contexts (which reads
              what was accepted), then ``BeamPool.truncate`` back to where the pass began.

The caches are beam trees: ``beams`` traces over a shared prompt, and after every ``interval`` tokens half of
them give way to branches of others, which share their parent's pages.  Shapes (lengths, trees, forks) come from
the case, values from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NO = -1e30           # below every score; exp of it is 0


# --------------------------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------------------------

def _prompt(name, **kw):
    c = {"name": name, "kind": "prompt", "dtype": "bf16", "seqs": 1, "shortest": 8192, "longest": 8192,
         "q_heads": 32, "kv_heads": 8, "head_dim": 128, "fused": True, "shape": 1}
    c.update(kw)
    return c


def _draft(name, **kw):
    c = {"name": name, "kind": "draft", "dtype": "bf16", "slots": 64, "beams": 64, "prompt": 512, "context": 4000,
         "interval": 512, "tokens": 16, "ragged": True, "layers": 2, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page": 16, "shape": 1}
    c.update(kw)
    return c


def listed():
    return [
        # One short question, fp32, the smallest configuration's heads: latency only.
        _prompt("prompt_short_f32", dtype="f32", shortest=64, longest=64, q_heads=4, kv_heads=2, head_dim=64, fused=False),
        # A serving batch of fp32 prompts, odd lengths.
        _prompt("prompt_packed_f32", dtype="f32", seqs=8, shortest=33, longest=1100, q_heads=4, kv_heads=2, head_dim=64),
        # One ordinary question of a reasoning benchmark.
        _prompt("prompt_300", shortest=333, longest=333),
        # A batch of prompts of one token to 2K, read from the fused projection's rows.
        _prompt("prompt_packed", seqs=24, shortest=1, longest=2048),
        # The prompt of the long-context search and more.
        _prompt("prompt_8k"),
        # The longest prompt, eight query heads per KV head.
        _prompt("prompt_16k_g8", shortest=16384, longest=16384, q_heads=16, kv_heads=2, fused=False),
        # The smallest search's traces, fp32, five drafted tokens each: latency only.
        _draft("draft_8_f32", dtype="f32", slots=8, beams=8, prompt=64, context=250, interval=96, tokens=5, layers=1,
               q_heads=4, kv_heads=2, head_dim=64),
        # One long trace, a chain of four drafted tokens: few rows over a long cache.
        _draft("draft_single_20k", slots=1, beams=1, prompt=20000, context=20000, interval=0, tokens=4, ragged=False),
        # The ordinary search: 64 traces at 4K, trees of up to 16 drafted tokens.
        _draft("draft_64x4k"),
        # Many traces at 8K, eight drafted tokens, eight query heads per KV head, slots that hold no beam.
        _draft("draft_198x8k", slots=210, beams=198, context=8000, tokens=8, q_heads=32, kv_heads=4, layers=1),
        # A whole round of a small search: the launches and the page accounting count.
        _draft("round_13", kind="round", slots=16, beams=13, prompt=333, context=700, interval=150, tokens=8, layers=4,
               page=64),
        # A whole round with every layer of a 36-layer model over short contexts: the copying counts.
        _draft("round_36layers", kind="round", slots=128, beams=128, prompt=64, context=190, interval=100, tokens=12,
               layers=36),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "draft", "draft", "round"])
    f32 = rng.random() < 0.2
    kvh = rng.choice([1, 2, 4]) if f32 else rng.choice([2, 4, 8])
    heads = {"dtype": "f32" if f32 else "bf16", "q_heads": kvh * rng.choice([2, 4, 8]), "kv_heads": kvh,
             "head_dim": 64 if f32 else 128, "shape": rng.randrange(1, 1 << 30)}
    if kind == "prompt":
        c = _prompt("", seqs=_log(rng, 1, 32), shortest=1, longest=_log(rng, 1, 2000 if f32 else 16384),
                    fused=rng.random() < 0.5, **heads)
        if rng.random() < 0.4:
            c["seqs"] = 1
        if c["seqs"] == 1:
            c["shortest"] = c["longest"]
        # No more work, and no more scores of padded prompts, than the largest listed case.
        while c["seqs"] * c["q_heads"] * c["longest"] ** 2 > 16 * 16384 ** 2:
            c["seqs"], c["longest"] = max(1, c["seqs"] // 2), max(1, c["longest"] * 3 // 4)
            c["shortest"] = min(c["shortest"], c["longest"])
    else:
        c = _draft("", kind=kind, beams=_log(rng, 1, 24 if f32 else 200), prompt=_log(rng, 1, 4096), tokens=_log(rng, 1, 64),
                   ragged=rng.random() < 0.7, layers=rng.choice([1, 2, 4]), page=rng.choice([16, 32, 64]), **heads)
        c["slots"] = c["beams"] + rng.choice([0, 0, _log(rng, 1, 64)])
        c["interval"] = _log(rng, 64, 1024)
        c["context"] = c["prompt"] + rng.choice([0, c["interval"], 3 * c["interval"] + rng.randint(1, 63), _log(rng, 1, 6000)])
        if kind == "round":
            c["context"] = min(c["context"], c["prompt"] + 2 * c["interval"])
        while c["beams"] * c["context"] * c["layers"] * kvh * (c["tokens"] * c["q_heads"] // kvh + 64) > 1.2e9:
            c["tokens"] = max(1, c["tokens"] * 2 // 3)
            c["layers"] = 1
            c["beams"] = max(1, c["beams"] * 3 // 4)
        c["slots"] = max(c["beams"], min(c["slots"], c["beams"] + 64))
    return c


def _lengths(case):
    """The prompts' lengths: spread over their logarithm, the longest among them."""
    rng = np.random.RandomState(case["shape"])
    lo, hi = math.log(case["shortest"]), math.log(case["longest"])
    n = np.exp(rng.uniform(lo, hi, case["seqs"])).round().astype(np.int64)
    n[rng.randint(case["seqs"])] = case["longest"]
    return n


def _grow(case):
    """The beams' contexts: (rows of the token store by beam and position, rounds), a round being
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


def _trees(case, salt):
    """(parent [slots][tokens], count [slots], accepted [slots]): drafted trees, each token a child of an earlier
    one or of the context, two in three continuing the one before."""
    rng = np.random.RandomState(case["shape"] ^ salt)
    slots, t = case["slots"], case["tokens"]
    i = np.arange(t)
    other = (rng.randint(0, 1 << 30, (slots, t)) % (i + 1)) - 1
    parent = np.where(rng.rand(slots, t) < 0.67, i - 1, other)
    count = rng.randint((t + 1) // 2, t + 1, slots) if case["ragged"] else np.full(slots, t)
    accepted = np.where(rng.rand(slots) < 0.1, -1, rng.randint(0, 1 << 30, slots) % count)
    return parent.astype(np.int32), count.astype(np.int32), accepted.astype(np.int32)


# --------------------------------------------------------------------------------------------
# What a program has before the call
# --------------------------------------------------------------------------------------------

def _rand(g, *shape, dtype=torch.bfloat16):
    """N(0, 1) values, drawn in parts where there are many."""
    if math.prod(shape) <= 1 << 28 or dtype == torch.float32:
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, hq, hkv, d = DT[case["dtype"]], case["q_heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case, "scale": 1 / math.sqrt(d)}
    if case["kind"] == "prompt":
        lengths = _lengths(case)
        total = int(lengths.sum())
        if case["fused"]:  # one projection's rows: q heads, then k heads, then v heads
            x = _rand(g, total, (hq + 2 * hkv) * d, dtype=dt)
            s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, d)) for t in x.split([hq * d, hkv * d, hkv * d], 1))
        else:
            s["q"], s["k"], s["v"] = (_rand(g, total, h, d, dtype=dt) for h in (hq, hkv, hkv))
        s["cu"] = torch.tensor(np.concatenate([[0], lengths.cumsum()]), dtype=torch.int32, device="cuda")
        s["longest"] = int(lengths.max())
        if own:
            from paper_2608_08020_gb300.prompt import PromptAttention
            s["op"] = PromptAttention(hq, hkv, d, case["dtype"], max_tokens=total, max_seqs=case["seqs"])
        return s
    rows, used, rounds = _grow(case)
    slots, beams, layers, t = case["slots"], case["beams"], case["layers"], case["tokens"]
    s["k"], s["v"] = (_rand(g, layers, used, hkv, d, dtype=dt) for _ in range(2))
    s["rows"] = torch.from_numpy(rows).cuda()
    for n, salt in (("1", 0x51), ("2", 0x52)) if case["kind"] == "round" else (("1", 0x51),):
        for x, h in (("q", hq), ("kd", hkv), ("vd", hkv)):
            s[x + n] = _rand(g, layers, slots, t, h, d, dtype=dt)
        s["parent" + n], s["count" + n], accepted = (torch.from_numpy(x).cuda() for x in _trees(case, salt))
        if n == "1":
            s["accepted"] = accepted
    if own:
        from paper_2608_08020_gb300.draft import DraftTrees
        from paper_2608_08020_gb300.pool import BeamPool
        width = -(-(case["context"] + t) // case["page"]) + 1
        pool = BeamPool(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=case["page"],
                        kv_dtype=case["dtype"], num_pages=used // case["page"] + (2 * len(rounds) + 8) * beams + 64,
                        max_beams=slots, max_pages_per_beam=width)
        p = case["prompt"]
        pool.seed(beams, p, s["k"][:, :p].contiguous(), s["v"][:, :p].contiguous())
        for _, n, first, parents in rounds:   # the store holds a round's rows beam by beam
            for j in range(0, n, 256):
                m = min(256, n - j)
                for layer in range(layers):
                    x = torch.zeros(2, m, slots, hkv, d, dtype=dt, device="cuda")
                    for kv, store in enumerate((s["k"], s["v"])):
                        x[kv, :, :beams] = store[layer, first:first + beams * n].unflatten(0, (beams, n))[:, j:j + m].transpose(0, 1)
                    pool.append_kv(layer, m, x[0], x[1])
            if parents is not None:
                pf = np.full(slots, -1, np.int32)
                pf[:beams] = parents
                pool.fork_slots(torch.from_numpy(pf).cuda())
        assert pool.status() == 0
        s["pool"], s["trees"] = pool, DraftTrees(pool, t)
        s["start"] = torch.full((slots,), case["context"], dtype=torch.int32, device="cuda")
    return s


# --------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------

def run(s):
    kind, layers = s["case"]["kind"], s["case"]["layers"] if "layers" in s["case"] else 0
    if kind == "prompt":
        return s["op"](s["q"], s["k"], s["v"], s["cu"], s["scale"]) if own else _plain_prompt(s)
    if not own:
        return _plain_draft(s)
    trees = s["trees"]
    if kind == "draft":
        return [trees.attention(i, s["q1"][i], s["kd1"][i], s["vd1"][i], s["parent1"], s["scale"], count=s["count1"])
                for i in range(layers)]
    n, path = trees.accept(s["kd1"], s["vd1"], s["parent1"], s["accepted"], count=s["count1"])
    out = [trees.attention(i, s["q2"][i], s["kd2"][i], s["vd2"][i], s["parent2"], s["scale"], count=s["count2"])
           for i in range(layers)]
    s["pool"].truncate(s["start"])
    return {"n": n, "path": path, "out": out}


def _softmax(x):
    """Softmax over the last axis, in place; scores of NO count as absent."""
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    return x.div_(x.sum(-1, keepdim=True))


def _plain_prompt(s):
    """Prompts padded to the longest one, all their scores at once, in 32 bits."""
    q, k, v, cu, most = s["q"], s["k"], s["v"], s["cu"].long(), s["longest"]
    hq, hkv, d = q.shape[1], k.shape[1], q.shape[2]
    t = torch.arange(most, device=q.device)
    there = t < (cu[1:] - cu[:-1])[:, None]                                       # [seqs][most]
    at = (cu[:-1, None] + t).clamp_(max=q.shape[0] - 1)
    qp = q[at].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4)      # [seqs][hkv][G][most][d]
    kp, vp = k[at].float().permute(0, 2, 3, 1), v[at].float().transpose(1, 2)
    x = torch.matmul(qp.flatten(2, 3), kp).mul_(s["scale"]).unflatten(2, (hq // hkv, most))
    x.masked_fill_(t > t[:, None], NO)
    o = torch.matmul(_softmax(x).flatten(2, 3), vp).unflatten(2, (hq // hkv, most))
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[there].to(q.dtype)


def _ancestors(parent, count):
    """[slots][tokens][tokens]: whether token j is token i or one of its ancestors (both among the first `count`)."""
    i = torch.arange(parent.shape[1], device=parent.device)
    a = ((parent[:, :, None] == i) | (i[:, None] == i)).float()
    for _ in range(6):      # paths of up to 64 tokens, doubled each time
        a = (torch.matmul(a, a) > 0).float()
    here = i < count[:, None]
    return (a > 0) & here[:, :, None] & here[:, None, :]


def _plain_draft(s):
    """Every beam's context gathered, then the drafted rows beside it, in 32 bits.  In a round the drafts accepted
    first are the rows of their tree that lie on the path."""
    case, rows = s["case"], s["rows"]
    beams, t, hkv = case["beams"], case["tokens"], case["kv_heads"]
    last = "2" if case["kind"] == "round" else "1"
    q, parent, count = s["q" + last], s["parent" + last], s["count" + last].long()
    keys = [s["k"][:, rows], s["kd" + last][:, :beams]]
    vals = [s["v"][:, rows], s["vd" + last][:, :beams]]
    sees = _ancestors(parent, count)
    seen = [torch.ones(beams, t, rows.shape[1], dtype=torch.bool, device=q.device), sees[:beams]]
    if last == "2":
        acc, first = s["accepted"].long(), _ancestors(s["parent1"], s["count1"].long())
        on = first[torch.arange(len(acc), device=q.device), acc.clamp(min=0)] & (acc >= 0)[:, None]
        on[beams:] = False
        keys.insert(1, s["kd1"][:, :beams])
        vals.insert(1, s["vd1"][:, :beams])
        seen.insert(1, on[:beams, None].expand(-1, t, -1))
    k, v = torch.cat(keys, 2).float().permute(0, 1, 3, 4, 2), torch.cat(vals, 2).float().transpose(2, 3)
    seen = torch.cat(seen, 2)[:, None, :, None]                                    # [beams][1][t][1][keys]
    g = q.shape[3] // hkv
    x = q[:, :beams].float().unflatten(3, (hkv, g)).transpose(2, 3)                # [layers][beams][hkv][t][g][d]
    x = torch.matmul(x.flatten(3, 4), k).mul_(s["scale"]).unflatten(3, (t, g))
    x.masked_fill_(~seen, NO)
    o = torch.matmul(_softmax(x).flatten(3, 4), v).unflatten(3, (t, g)).transpose(2, 3).flatten(3, 4)
    out = torch.zeros_like(q)
    out[:, :beams] = torch.where((torch.arange(t, device=q.device) < count[:beams, None])[:, :, None, None], o, 0).to(q.dtype)
    if last == "1":
        return list(out)
    i = torch.arange(t, device=q.device)
    n = on.sum(1)
    path = torch.where(on, i, t).sort(1).values
    return {"n": n.int(), "path": torch.where(i < n[:, None], path, -1).int(), "out": list(out)}


# --------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------

def work(case):
    hq, hkv, d, es = case["q_heads"], case["kv_heads"], case["head_dim"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "prompt":
        n = _lengths(case).astype(np.float64)
        # q, k, v read once, the output written once; row i has i + 1 keys.
        return {"bytes": float(n.sum()) * (2 * hq + 2 * hkv) * d * es, "flops": float((n * (n + 1) / 2).sum()) * hq * 4 * d}
    beams, layers = case["beams"], case["layers"]
    rows, _, _ = _grow(case)
    seen = float(np.unique(rows).size)                   # tokens some beam still holds, each read once
    last = 0x52 if case["kind"] == "round" else 0x51
    parent, count, _ = _trees(case, last)
    depth = np.zeros((beams, case["tokens"]))
    for i in range(case["tokens"]):
        up = parent[:beams, i]
        depth[:, i] = 1 + np.where(up >= 0, depth[np.arange(beams), np.maximum(up, 0)], 0)
    here = np.arange(case["tokens"]) < count[:beams, None]
    drafted = float(here.sum())
    keys = float((np.where(here, depth, 0)).sum()) + drafted * case["context"]
    b = (seen + drafted) * 2 * hkv * d * es + drafted * hq * d * es + case["slots"] * case["tokens"] * hq * d * es
    if case["kind"] == "round":
        n, _ = _path(case)
        taken = float(sum(n))
        b += taken * 3 * 2 * hkv * d * es                # read among the drafts, written to the cache, read by the attention
        keys += float((here.sum(1) * np.array(n)).sum())
    return {"bytes": layers * b, "flops": layers * keys * hq * 4 * d}


def _path(case):
    """Each beam's accepted path, walked up from its last token."""
    parent, _, accepted = _trees(case, 0x51)
    paths = []
    for b in range(case["beams"]):
        p, i = [], int(accepted[b])
        while i >= 0:
            p.insert(0, i)
            i = int(parent[b, i])
        paths.append(p)
    return [len(p) for p in paths], paths


# --------------------------------------------------------------------------------------------
# The definition, in 64 bits
# --------------------------------------------------------------------------------------------

def _attend(q, k, v, scale, sees=None):
    """q [t][hq][d] over k, v [keys][hkv][d]: softmax(scale q.k) v by query head, keys where sees [t][keys]."""
    g = q.shape[1] // k.shape[1]
    o = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for h in range(q.shape[1]):
        x = q[:, h].double() @ k[:, h // g].double().T * scale
        if sees is not None:
            x = x.masked_fill(~sees, -math.inf)
        o[:, h] = torch.softmax(x, -1) @ v[:, h // g].double()
    return o


def exact(case, seed):
    if work(case)["flops"] > 1.5e12:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "prompt":
        out, at = [], s["cu"].tolist()
        for a, b in zip(at, at[1:]):
            for r in range(a, b, 2048):     # rows of a long prompt in parts, each over the keys up to its end
                e = min(b, r + 2048)
                sees = torch.arange(e - a, device="cuda") <= torch.arange(r - a, e - a, device="cuda")[:, None]
                out.append(_attend(s["q"][r:e], s["k"][a:e], s["v"][a:e], s["scale"], sees))
        return torch.cat(out)
    last = "2" if case["kind"] == "round" else "1"
    parent, count = s["parent" + last].tolist(), s["count" + last].tolist()
    n, paths = _path(case) if last == "2" else (None, [[]] * case["beams"])
    out = [torch.zeros(s["q1"].shape[1:], dtype=torch.float64, device="cuda") for _ in range(case["layers"])]
    for b in range(case["beams"]):
        c = count[b]
        sees = torch.zeros(c, c, dtype=torch.bool)
        for i in range(c):
            j = i
            while j >= 0:
                sees[i, j] = True
                j = parent[b][j]
        before = case["context"] + len(paths[b])
        sees = torch.cat([torch.ones(c, before, dtype=torch.bool), sees], 1).cuda()
        for layer in range(case["layers"]):
            kv = []
            for x in ("k", "v"):
                parts = [s[x][layer, s["rows"][b]], s[x + "d" + last][layer, b, :c]]
                if paths[b]:
                    parts.insert(1, s[x + "d1"][layer, b, paths[b]])
                kv.append(torch.cat(parts))
            out[layer][b, :c] = _attend(s["q" + last][layer, b, :c], kv[0], kv[1], s["scale"], sees)
    return out if last == "1" else {"n": None, "path": None, "out": out}
