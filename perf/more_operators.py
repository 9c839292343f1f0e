"""The calls on a paged key/value cache held in 4 bits whose time matters, with their inputs, plain forms and exact values.

Three operators: ``store`` (keys and values quantised as they are written, and read back as what they have become, which is
what the prompt's own attention has to see if it is to see what later tokens will), ``read`` (cached tokens as 16-bit floats, from
their pages in order: requests that leave the accelerator, or are looked at) and ``attend`` (attention over the pages).

A token's keys (values) of a head are cut into groups of 32, the last one shorter.  A group is kept as its lowest value
``lo``, a step and 4 bits for each value x:
  step   the largest 16-bit float of the cache's type that is not above (max - lo) / 15; the smallest positive one
         where that is 0 and max is not lo,
  code   (x - lo) / step rounded to the nearest of 0 .. 15, ties to even; 0 where step is 0,
and the cache holds the 16-bit float nearest to lo + code step in x's place.  The table, lengths and references are those
of the 16-bit cache.  Lengths follow from the case alone; values and the pages' order from the seed.
"""
import math
import random

import numpy as np
import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
GROUP = 32


def listed():
    A = dict(op="attend", groups=0, prefix=0, q_lo=1, q_hi=1, write=False)
    R = dict(op="read", tail=0)
    return [
        # One step of the 50-request instance (M = 2000): some 40 short sequences, where the calls' latency counts.
        dict(A, name="attend_50", dtype="bf16", kv_heads=8, group=4, dim=128, page=16, n=40, own_lo=2, own_hi=98),
        # A layer of one step of the 1000-request instances (M = 16384): the new tokens written, then attention; small heads, float16.
        dict(A, name="layer_thousand", dtype="f16", kv_heads=8, group=2, dim=64, page=16, n=64, own_lo=1, own_hi=512, write=True),
        # One step of the 10^5-request streams (M = 500000): the memory-bound step of a full accelerator.
        dict(A, name="attend_online", dtype="bf16", kv_heads=8, group=8, dim=128, page=64, n=384, own_lo=1, own_hi=2600),
        # One request over a long document: a single row of queries per head, so the keys have to be split.
        dict(A, name="attend_long", dtype="f16", kv_heads=8, group=8, dim=128, page=32, n=1, own_lo=131071, own_hi=131071),
        # A batch under one system prompt: 256 sequences forked from it, each with some tokens of its own.
        dict(A, name="prefix_batch", dtype="bf16", kv_heads=8, group=8, dim=128, page=16, n=256, own_lo=1, own_hi=512,
             groups=1, prefix=8192),
        # Several ragged groups (samples of one prompt each), odd head counts, drafted tokens beside single ones.
        dict(A, name="prefix_groups", dtype="f16", kv_heads=3, group=5, dim=80, page=32, n=61, own_lo=5, own_hi=300,
             groups=7, prefix=2000, q_lo=1, q_hi=5),
        # The prompts' own parts after a shared prefix, many tokens at once: bound by the matrix products.
        dict(A, name="prefix_prefill", dtype="bf16", kv_heads=8, group=8, dim=128, page=64, n=16, own_lo=512, own_hi=700,
             groups=1, prefix=4096, q_lo=300, q_hi=512),
        # A token for each of some 40 sequences.
        dict(op="store", name="store_step_50", dtype="bf16", kv_heads=8, dim=128, page=16, n=40, own_lo=1, own_hi=1),
        # Prompts of the 10^5-request streams admitted at once.
        dict(op="store", name="store_admit", dtype="bf16", kv_heads=8, dim=128, page=16, n=250, own_lo=1, own_hi=2048),
        # Prompts of many lengths, odd heads and sizes, float16.
        dict(op="store", name="store_ragged", dtype="f16", kv_heads=3, dim=80, page=32, n=77, own_lo=1, own_hi=3000),
        # The last tokens of each sequence: what a request that is cancelled and goes on elsewhere takes along.
        dict(R, name="read_tail", dtype="f16", kv_heads=4, dim=64, page=32, n=40, own_lo=1, own_hi=600, tail=37),
        # Whole sequences that leave the accelerator to make room.
        dict(R, name="read_evict", dtype="bf16", kv_heads=8, dim=128, page=64, n=96, own_lo=1, own_hi=4000),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.5 / hi))))


def draw(rng):
    dtype, page, dim = rng.choice(sorted(DTYPES)), rng.choice([16, 32, 64, 128]), rng.choice([32, 64, 80, 96, 128])
    heads, op = rng.choice([1, 2, 3, 4, 8]), rng.choice(["attend", "attend", "attend", "store", "read"])
    if op == "attend":
        c = dict(op=op, dtype=dtype, kv_heads=heads, group=rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), dim=dim, page=page, n=_log(rng, 1, 400),
                 own_lo=1, own_hi=_log(rng, 1, 4096), groups=0, prefix=0, q_lo=1, q_hi=1, write=rng.random() < 0.3)
        if rng.random() < 0.5:
            c.update(groups=rng.randint(1, max(1, min(8, c["n"] // 2))), prefix=_log(rng, 100, 8192))
        if rng.random() < 0.4:
            c.update(q_hi=_log(rng, 2, 300))
            c.update(n=min(c["n"], 32), own_lo=c["q_hi"], own_hi=c["own_hi"] + c["q_hi"])
        # what the plain form gathers, and its products, stay below those of the largest listed cases
        keys = (c["prefix"] + c["own_hi"]) * heads
        c["n"] = max(1, min(c["n"], 8_000_000 // keys, 2_400_000_000 // (keys * c["group"] * c["q_hi"])))
        c["groups"] = min(c["groups"], c["n"])
        return c
    n = _log(rng, 1, 250)
    c = dict(op=op, dtype=dtype, kv_heads=heads, dim=dim, page=page, n=n, own_lo=1, own_hi=_log(rng, 1, min(4000, 250_000 // n)))
    if op == "read":
        c.update(tail=rng.choice([0, _log(rng, 1, 500)]))
    return c


def _shape(c):
    """Lengths, queries and groups of a case: they follow from its values alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    n = c["n"]
    q = [rng.randint(c.get("q_lo", 1), c.get("q_hi", 1)) for _ in range(n)]
    mine = [max(rng.randint(c["own_lo"], c["own_hi"]), x) for x in q]
    g = c.get("groups", 0)
    cuts = sorted(rng.sample(range(1, n), g - 1)) if g else []
    bounds = [0, *cuts, n] if g else list(range(n + 1))
    pre = [rng.randint(c["prefix"] * 3 // 4, c["prefix"]) if g else 0 for _ in bounds[1:]]
    return q, mine, bounds, pre


def _groups(dim):
    return -(-dim // GROUP)


def work(case):
    q, mine, bounds, pre = _shape(case)
    P, D, H = case["page"], case["dim"], case["kv_heads"]
    held, whole = 2 * H * (D // 2 + 4 * _groups(D)), 4 * H * D  # bytes of a token's keys and values: in the cache, as 16-bit floats
    if case["op"] == "attend":
        keys = sum(pre) + sum(mine)  # each key and value once: a prefix for all of its group
        hq = H * case["group"]
        of = [p for p, a, b in zip(pre, bounds, bounds[1:]) for _ in range(b - a)]
        seen = sum(x * (p + m) - x * (x - 1) // 2 for x, p, m in zip(q, of, mine))
        new = sum(q) * whole if case["write"] else 0
        return {"bytes": keys * held + new + sum(q) * hq * (D * 4 + 4) + 4 * (keys // P + 2 * len(q)), "flops": 4 * seen * hq * D}
    tokens = sum(min(m, case["tail"]) if case.get("tail") else m for m in mine)
    stored = case["op"] == "store"
    return {"bytes": tokens * (held + whole + (whole + 8 if stored else 0)) + 4 * (tokens // P + 2 * len(mine)),
            "flops": tokens * H * D * (16 if stored else 4)}


def _inputs(c, seed):
    """What both forms are given: the tables, what the pages hold (16-bit floats, not yet quantised), queries or tokens to write."""
    dev = "cuda"
    gen = torch.Generator(dev).manual_seed(seed)
    host = np.random.default_rng(seed)
    q, mine, bounds, pre = _shape(c)
    P, D, H, n, dt = c["page"], c["dim"], c["kv_heads"], c["n"], DTYPES[c["dtype"]]
    of = [p for p, a, b in zip(pre, bounds, bounds[1:]) for _ in range(b - a)]
    n_pages = sum(p // P for p in pre) + sum(-(-(p + m) // P) - p // P for p, m in zip(of, mine)) + 7
    most = max(-(-(p + m) // P) for p, m in zip(of, mine)) + 3
    order = host.permutation(n_pages).astype(np.int32)  # pages in use lie anywhere after some time
    table, length, ref = np.full((n, most), -1, np.int32), np.zeros(n, np.int32), np.zeros(n_pages, np.int32)
    at = 0

    def take(k):
        nonlocal at
        at += k
        return order[at - k:at]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    for p, a, b in zip(pre, bounds, bounds[1:]):
        first = take(p // P)
        for i in range(a, b):
            length[i] = p + mine[i]
            k = -(-int(length[i]) // P)
            table[i, : p // P] = first
            table[i, p // P: k] = take(k - p // P)
    np.add.at(ref, table[table >= 0], 1)
    # Keys have channels that are far from zero in all tokens, values tokens that are larger than others.
    bias = torch.empty(H, 1, D, device=dev).normal_(generator=gen)
    bias *= torch.where(torch.rand(H, 1, D, device=dev, generator=gen) < 0.04, 6.0, 1.0)

    def values(*shape):
        x = torch.empty(*shape, dtype=dt, device=dev).normal_(generator=gen)
        return x, torch.empty(*shape[:-1], 1, dtype=dt, device=dev).normal_(generator=gen).mul_(0.5).exp_()

    s = dict(c=c, table=ints(table), length=ints(length), ref=ints(ref), seqs=ints(range(n)), n_pages=n_pages)
    if c["op"] != "store":
        x, size = values(n_pages, 2, H, P, D)
        x[:, 0] += bias.to(dt)
        x[:, 1] *= size[:, 1]
        s["pool"] = x
    slots_of = [table[i, (length[i] - t + np.arange(t)) // P].astype(np.int64) * P + (length[i] - t + np.arange(t)) % P
                for i, t in enumerate(mine if c["op"] == "store" else q)]
    if c["op"] == "attend":
        n_q = sum(q)
        x = torch.empty(n_q, H * c["group"], D, dtype=dt, device=dev).normal_(generator=gen)
        s.update(q=x, cu_q=ints([0, *np.cumsum(q)]), n_q=n_q, max_q=max(q), max_len=int(length.max()), cu_group=ints(bounds) if c["groups"] else None)
    if c["op"] == "store" or c.get("write"):
        s["slots"] = torch.from_numpy(np.concatenate(slots_of)).to(dev)
        total = s["slots"].numel()
        k, _ = values(total, H, D)
        v, size = values(total, H, D)
        s.update(k=k + bias.to(dt).view(1, H, D), v=v * size)
    if c["op"] != "attend":
        count = [min(m, c["tail"]) if c.get("tail") else m for m in mine]
        s.update(cu=ints([0, *np.cumsum(count)]), total=sum(count), first=ints([m - x for m, x in zip(mine, count)]) if c.get("tail") else None)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    pool, P, H, D, dt = s.pop("pool", None), case["page"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    step = 1 + 40_000_000 // (H * P * D)  # pages quantised at a time
    if own:
        from paper_2508_14544_gb300 import KVCache
        kv = KVCache(s["n_pages"], P, H, D, *s["table"].shape, dtype=dt, bits=4)
        kv.table.copy_(s["table"])
        kv.length.copy_(s["length"])
        kv.ref.copy_(s["ref"])
        for a in range(0, s["n_pages"] if pool is not None else 0, step):
            x = pool[a: a + step].transpose(2, 3)
            rows = torch.arange(a * P, a * P + x.shape[0] * P, device="cuda")
            kv.write(rows, x[:, 0].reshape(-1, H, D), x[:, 1].reshape(-1, H, D))
        s["cache"] = kv
        if case.get("write"):
            s["plan"] = kv.plan(s["seqs"], s["cu_q"], s["n_q"], heads=s["q"].shape[1], cu_group=s["cu_group"])
    else:
        s["codes"] = torch.zeros(s["n_pages"], 2, H, P, D // 2, dtype=torch.uint8, device="cuda")
        s["scale"] = torch.zeros(s["n_pages"], 2, H, P, _groups(D), 2, dtype=dt, device="cuda")  # lo, step
        for a in range(0, s["n_pages"] if pool is not None else 0, step):
            s["codes"][a: a + step], s["scale"][a: a + step] = _quantise(pool[a: a + step])
    return s


# ---- plain forms: elementary operations on the whole batch, in 32 bits; in 64 for the steps and codes, which have borders ------

def _quantise(x):
    """Codes, two to a byte (the even place low), and lo and step of each group, of 16-bit floats [.., D]."""
    codes, scale = [], []
    for a in range(0, x.shape[-1], GROUP):
        y = x[..., a: a + GROUP].double()
        lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
        most = (hi - lo) / torch.full_like(lo, 15)  # not by a number, which would be multiplied by 1 / 15
        step = most.to(x.dtype)
        step = torch.where(step.double() > most, (step.view(torch.int16) - 1).view(x.dtype), step)  # of positive floats: the one below
        step = torch.where((step == 0) & (hi > lo), torch.ones_like(step, dtype=torch.int16).view(x.dtype), step)
        code = torch.round((y - lo) / torch.where(step == 0, 1.0, step.double())).clamp_(0, 15).to(torch.uint8)
        codes.append(code[..., ::2] | code[..., 1::2] << 4)
        scale.append(torch.cat([lo.to(x.dtype), step], -1))
    return torch.cat(codes, -1), torch.stack(scale, -2)


def _values(codes, scale):
    """The 16-bit floats that they stand for."""
    D = 2 * codes.shape[-1]
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    wide = scale.float().repeat_interleave(GROUP, -2)[..., :D, :]
    return (code.float() * wide[..., 1] + wide[..., 0]).to(scale.dtype)


def _plain_write(s):
    P = s["c"]["page"]
    page, off = s["slots"] // P, s["slots"] % P
    for v, x in enumerate((s["k"], s["v"])):
        s["codes"][page, v, :, off], s["scale"][page, v, :, off] = _quantise(x)


def _plain_read(s):
    P, cu = s["c"]["page"], s["cu"].long()
    i = torch.repeat_interleave(torch.arange(s["seqs"].numel(), device="cuda"), cu[1:] - cu[:-1])
    pos = torch.arange(s["total"], device="cuda") - cu[i]
    if s["first"] is not None:
        pos = pos + s["first"].long()[i]
    page, off = s["table"][s["seqs"].long()[i], pos // P].long(), pos % P
    return {x: _values(s["codes"][page, v, :, off], s["scale"][page, v, :, off]) for v, x in enumerate("kv")}


def _plain_attend(s):
    q, P, H, D, dev = s["q"], s["c"]["page"], s["c"]["kv_heads"], s["c"]["dim"], s["q"].device
    seqs, cu, n = s["seqs"].long(), s["cu_q"].long(), s["seqs"].numel()
    G, mq = q.shape[1] // H, s["max_q"]
    length, nq = s["length"][seqs].long(), cu[1:] - cu[:-1]
    pos = torch.arange(s["max_len"], device=dev)
    page = s["table"][seqs][:, pos // P].long().clamp(min=0)
    off = (pos % P)[None].expand_as(page)

    def cached(v):
        return _values(s["codes"][page, v, :, off], s["scale"][page, v, :, off]).float()  # [n, tokens, H, D]

    at = (cu[:-1, None] + torch.arange(mq, device=dev)[None]).clamp(max=max(s["n_q"] - 1, 0))
    x = q[at].float().view(n, mq, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, mq * G, D)
    sc = torch.matmul(x, cached(0).permute(0, 2, 3, 1)) * D ** -0.5
    last = length[:, None] - nq[:, None] + torch.arange(mq, device=dev)[None]
    hid = pos[None, None] > last[:, :, None]
    sc = sc.view(n, H, mq, G, -1).masked_fill_(hid[:, None, :, None], float("-inf"))
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, H, mq * G, -1), cached(1).permute(0, 2, 1, 3)).view(n, H, mq, G, D) / total.clamp(min=1e-38)
    lse = (m + total.log()).squeeze(-1)
    t = torch.arange(s["n_q"], device=dev)
    i = torch.searchsorted(cu[1:], t, right=True)
    j = t - cu[i]
    return {"out": o[i, :, j].reshape(-1, H * G, D).to(q.dtype), "lse": lse[i, :, j].reshape(-1, H * G)}


def run(s):
    op = s["c"]["op"]
    if not own:
        if op == "store" or s["c"].get("write"):
            _plain_write(s)
        return _plain_attend(s) if op == "attend" else _plain_read(s)
    kv = s["cache"]
    if op == "store" or s["c"].get("write"):
        kv.write(s["slots"], s["k"], s["v"])
    if op == "attend":
        plan = s["plan"] if s["c"]["write"] else kv.plan(s["seqs"], s["cu_q"], s["n_q"], heads=s["q"].shape[1], cu_group=s["cu_group"])
        out, lse = kv.attend(s["q"], plan)
        return {"out": out, "lse": lse}
    k, v = kv.read(s["seqs"], s["cu"], s["total"], first=s["first"])
    return {"k": k, "v": v}


# ---- from the definition, in 64 bits ---------------------------------------------------------------------------------

def _grid(x, dtype, down):
    """x >= 0 (down) or of any sign on the type's grid: the next one below, or the nearest, ties to even."""
    bits, least = {torch.bfloat16: (8, -133), torch.float16: (11, -24)}[dtype]
    e = torch.clamp(torch.frexp(x)[1] - bits, min=least).long()
    unit = ((e + 1023) << 52).view(torch.float64)  # 2^e; pow need not be exact
    y = x / unit
    return (torch.floor(y) if down else torch.round(y)) * unit


def _held(x):
    """What the cache holds in the place of 16-bit floats [.., D]."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    least = 2.0 ** {torch.bfloat16: -133, torch.float16: -24}[x.dtype]
    for a in range(0, x.shape[-1], GROUP):
        y = x[..., a: a + GROUP].to(torch.float64)
        lo = y.min(-1, keepdim=True).values
        span = y.max(-1, keepdim=True).values - lo
        step = torch.where(span > 0, _grid(span / torch.full_like(span, 15), x.dtype, True).clamp(min=least), 1.0)
        code = torch.clamp(torch.round((y - lo) / step), max=15)
        out[..., a: a + GROUP] = _grid(lo + code * step, x.dtype, False)
    return out


def exact(case, seed):
    """The values held, and attention over them a sequence at a time."""
    s = _inputs(case, seed)
    P, H, D = case["page"], case["kv_heads"], case["dim"]
    table = s["table"].cpu().numpy()
    if case["op"] == "store":
        return {"k": _held(s["k"]), "v": _held(s["v"])}
    pool, length = s["pool"], s["length"].tolist()
    if case.get("write"):
        for v, x in enumerate((s["k"], s["v"])):
            pool[s["slots"] // P, v, :, s["slots"] % P] = x

    def tokens(i, a, b):  # [2, H, b - a, D] of sequence i
        rows = torch.from_numpy(table[i, a // P: -(-b // P)].astype(np.int64)).cuda()
        x = pool[rows].permute(1, 2, 0, 3, 4).reshape(2, H, -1, D)
        return _held(x[:, :, a % P: a % P + b - a])

    if case["op"] == "read":
        first = [0] * len(length) if s["first"] is None else s["first"].tolist()
        parts = [tokens(i, a, b).transpose(1, 2) for i, (a, b) in enumerate(zip(first, length))]
        return {x: torch.cat([p[v] for p in parts]) for v, x in enumerate("kv")}
    cu, out, lse = s["cu_q"].tolist(), [], []
    for i, size in enumerate(length):
        kv = tokens(i, 0, size)
        x = s["q"][cu[i]: cu[i + 1]].double().unflatten(1, (H, -1))  # [t, H, G, D]
        t = x.shape[0]
        y = torch.einsum("thgd,hsd->htgs", x, kv[0]) / math.sqrt(D)
        seen = torch.arange(size, device="cuda")[None] <= torch.arange(size - t, size, device="cuda")[:, None]
        y = torch.where(seen[None, :, None], y, -math.inf)
        top = y.max(-1).values
        w = torch.exp(y - top[..., None])
        z = w.sum(-1)
        o = torch.einsum("htgs,hsd->htgd", w / z[..., None], kv[1])
        out.append(o.permute(1, 0, 2, 3).reshape(t, -1, D))
        lse.append((top + torch.log(z)).permute(1, 0, 2).reshape(t, -1))
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
