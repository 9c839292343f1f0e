"""The calls on a paged key/value cache whose time matters, with their inputs, plain forms and exact values.

Two operators: the pages themselves (``extend``, ``write``, ``fork``, ``copy``, ``free``, ``compact``: what
admission, generation, cancellation and completion of a request do to the memory that the schedulers count in
tokens), and attention of a batch's queries over the pages, in which sequences forked from one prefix read it
once for all.

The cache is ``pool`` [pages, layers, 2 (keys, values), kv_heads, page, dim], ``table`` int32 [sequences, pages per
sequence] (-1 where there is none), ``length`` int32 [sequences] and ``ref`` int32 [pages], the number of sequences
that hold a page (0: free).  Pages are given out lowest number first.  Lengths follow from the case alone; values
and the pages' order from the seed.
"""
import math
import random

import numpy as np
import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    A = dict(op="attend", groups=0, prefix=0, q_lo=1, q_hi=1)
    P = dict(op="pages", dtype="bf16")
    return [
        # One step of the 50-request instance (M = 2000): some 40 short sequences, where the calls' latency counts.
        dict(A, name="attend_50", dtype="bf16", kv_heads=8, group=4, dim=128, page=16, n=40, own_lo=2, own_hi=98),
        # One step of the 1000-request instances (M = 16384): short ragged sequences, small heads, float16.
        dict(A, name="attend_thousand", dtype="f16", kv_heads=8, group=2, dim=64, page=16, n=64, own_lo=1, own_hi=512),
        # One step of the 10^5-request streams (M = 500000): the memory-bound step of a full accelerator.
        dict(A, name="attend_online", dtype="bf16", kv_heads=8, group=8, dim=128, page=64, n=384, own_lo=1, own_hi=2600),
        # One request over a long document: a single row of queries per head, so the keys have to be split.
        dict(A, name="attend_long", dtype="bf16", kv_heads=8, group=8, dim=128, page=32, n=1, own_lo=131071, own_hi=131071),
        # A batch under one system prompt: 256 sequences forked from it, each with some tokens of its own.
        dict(A, name="prefix_batch", dtype="bf16", kv_heads=8, group=8, dim=128, page=16, n=256, own_lo=1, own_hi=512,
             groups=1, prefix=8192),
        # Several ragged groups (samples of one prompt each), odd head counts, drafted tokens beside single ones.
        dict(A, name="prefix_groups", dtype="f16", kv_heads=3, group=5, dim=80, page=32, n=61, own_lo=5, own_hi=300,
             groups=7, prefix=2000, q_lo=1, q_hi=5),
        # The prompts' own parts after a shared prefix, many tokens at once: bound by the matrix products.
        dict(A, name="prefix_prefill", dtype="bf16", kv_heads=8, group=8, dim=128, page=64, n=16, own_lo=512, own_hi=700,
             groups=1, prefix=4096, q_lo=300, q_hi=512),
        # One step of the 50-request instance: a token for each sequence, and its page where one is full.
        dict(P, name="pages_step_50", kind="step", layers=1, kv_heads=8, dim=128, page=16, n=40, own_lo=2, own_hi=98),
        # Prompts of the 10^5-request streams admitted at once: pages given out and one layer's keys and values written.
        dict(P, name="pages_admit", kind="admit", layers=1, kv_heads=8, dim=128, page=16, n=250, own_lo=1, own_hi=2048),
        # 256 samples of one prompt that ends inside a page: forked, the shared page copied at the first token.
        dict(P, name="pages_fork", kind="fork", layers=4, kv_heads=8, dim=128, page=16, n=256, own_lo=2041, own_hi=2041),
        # Sequences with pages of their own made from others (what is to be edited apart, not shared).
        dict(P, name="pages_copy", kind="copy", layers=2, kv_heads=4, dim=64, page=32, n=77, own_lo=1, own_hi=3000),
        # A quarter of the sequences ends, the holes are closed, and others are admitted at the end.
        dict(P, name="pages_churn", kind="churn", layers=4, kv_heads=8, dim=128, page=16, n=64, own_lo=900, own_hi=1100),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.5 / hi))))


def draw(rng):
    dtype = rng.choice(sorted(DTYPES))
    page = rng.choice([16, 32, 64, 128])
    if rng.random() < 0.6:
        c = dict(op="attend", dtype=dtype, kv_heads=rng.choice([1, 2, 3, 4, 8]), group=rng.choice([1, 2, 3, 4, 5, 7, 8, 16]),
                 dim=rng.choice([64, 80, 96, 128]), page=page, n=_log(rng, 1, 400), own_lo=1, own_hi=_log(rng, 1, 4096), groups=0,
                 prefix=0, q_lo=1, q_hi=1)
        if rng.random() < 0.6:
            c.update(groups=rng.randint(1, max(1, min(8, c["n"] // 2))), prefix=_log(rng, 100, 8192))
        if rng.random() < 0.4:
            c.update(q_hi=_log(rng, 2, 300))
            c.update(n=min(c["n"], 32), own_lo=c["q_hi"], own_hi=c["own_hi"] + c["q_hi"])
        # what the plain form gathers, and its products, stay below those of the largest listed cases
        keys = (c["prefix"] + c["own_hi"]) * c["kv_heads"]
        c["n"] = max(1, min(c["n"], 8_000_000 // keys, 2_400_000_000 // (keys * c["group"] * c["q_hi"])))
        c["groups"] = min(c["groups"], c["n"])
        return c
    return dict(op="pages", dtype=dtype, kind=rng.choice(["step", "admit", "fork", "copy", "churn"]), layers=rng.randint(1, 4),
                kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([64, 80, 96, 128]), page=page, n=_log(rng, 4, 250), own_lo=1,
                own_hi=_log(rng, 2, 1000))


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


def work(case):
    q, mine, bounds, pre = _shape(case)
    P, D, H = case["page"], case["dim"], case["kv_heads"]
    if case["op"] == "attend":
        keys = sum(pre) + sum(mine)  # each key and value once: a prefix for all of its group
        hq = H * case["group"]
        of = [p for p, a, b in zip(pre, bounds, bounds[1:]) for _ in range(b - a)]
        seen = sum(x * (p + m) - x * (x - 1) // 2 for x, p, m in zip(q, of, mine))
        return {"bytes": keys * H * D * 4 + sum(q) * hq * (D * 4 + 4) + 4 * (keys // P + 2 * len(q)), "flops": 4 * seen * hq * D}
    token, pages = 4 * H * D, [-(-m // P) for m in mine]  # bytes of one layer's keys and values; pages of each sequence
    whole, entries = token * P * case["layers"], sum(pages)
    if case["kind"] == "step":
        moved = 2 * len(mine) * token
    elif case["kind"] == "admit":
        moved = 2 * sum(mine) * token
    elif case["kind"] == "fork":
        entries = len(mine) * pages[0]
        moved = 2 * len(mine) * token + (len(mine) + 1) * whole * (mine[0] % P != 0)
    elif case["kind"] == "copy":
        moved = 2 * entries * whole
    else:
        moved = 2 * whole * sum(pages[: len(mine) // 4])
    return {"bytes": moved + 16 * entries, "flops": entries}


def _case_pages(c):
    """Pages of the pool, sequences, and pages that a row of the table has room for."""
    q, mine, bounds, pre = _shape(c)
    P = c["page"]
    if c["op"] == "attend":
        of = [p for p, a, b in zip(pre, bounds, bounds[1:]) for _ in range(b - a)]
        used = sum(p // P for p in pre) + sum(-(-(p + m) // P) - p // P for p, m in zip(of, mine))
        return used + 7, len(mine), max(-(-(p + m) // P) for p, m in zip(of, mine)) + 3
    most = max(-(-m // P) for m in mine) + 2
    used = sum(-(-m // P) for m in mine)
    if c["kind"] == "fork":
        return most + len(mine) * 2 + 9, len(mine) + 1, most
    if c["kind"] == "copy":
        return 2 * used + 9, 2 * len(mine), most
    return used + len(mine) + 9, len(mine), most


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(dev).manual_seed(seed)
    host = np.random.default_rng(seed)
    q, mine, bounds, pre = _shape(c)
    P, D, H, n = c["page"], c["dim"], c["kv_heads"], c["n"]
    n_pages, n_seq, most = _case_pages(c)
    dt = DTYPES[c["dtype"]]
    pool = torch.empty(n_pages, c.get("layers", 1), 2, H, P, D, dtype=dt, device=dev)
    pool.normal_(generator=gen)
    order = host.permutation(n_pages).astype(np.int32)  # pages in use lie anywhere after some time
    table, length, ref = np.full((n_seq, most), -1, np.int32), np.zeros(n_seq, np.int32), np.zeros(n_pages, np.int32)
    at = 0

    def take(k):
        nonlocal at
        at += k
        return order[at - k:at]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    s = {}
    if c["op"] == "attend":
        for p, a, b in zip(pre, bounds, bounds[1:]):
            first = take(p // P)
            for i in range(a, b):
                length[i] = p + mine[i]
                k = -(-int(length[i]) // P)
                table[i, : p // P] = first
                table[i, p // P: k] = take(k - p // P)
        n_q = sum(q)
        x = torch.empty(n_q, H * c["group"], D, dtype=dt, device=dev).normal_(generator=gen)
        s.update(q=x, seqs=ints(range(n)), cu_q=ints([0, *np.cumsum(q)]), n_q=n_q, max_q=max(q), max_len=int(length.max()),
                 cu_group=ints(bounds) if c["groups"] else None)
    else:
        new = [1] * n
        if c["kind"] in ("step", "copy", "churn"):
            for i in range(n):
                length[i] = mine[i]
                table[i, : -(-mine[i] // P)] = take(-(-mine[i] // P))
            if c["kind"] == "churn":
                new = [mine[0]] * n
        elif c["kind"] == "fork":
            length[n] = mine[0]
            table[n, : -(-mine[0] // P)] = take(-(-mine[0] // P))
        else:
            new = mine
        if c["kind"] in ("step", "admit", "fork"):
            s.update(k=torch.empty(sum(new), H, D, dtype=dt, device=dev).normal_(generator=gen))
            s.update(v=torch.empty(sum(new), H, D, dtype=dt, device=dev).normal_(generator=gen))
        s.update(seqs=ints(range(n)), cu_new=ints([0, *np.cumsum(new)]), total=sum(new), keep=ints(length[:n].copy()), src=ints([n] * n),
                 dst=ints(range(n, 2 * n)), turn=0, quarter=max(1, n // 4))
        if c["kind"] == "churn":  # the requests that end and come in are lists that the scheduler holds
            k = s["quarter"]
            parts = [list(range(a, min(a + k, n))) for a in range(0, n, k)]
            s.update(parts=[(ints(p), ints([0, *np.cumsum([mine[i] for i in p])]), sum(mine[i] for i in p)) for p in parts])
    held = table[table >= 0]
    np.add.at(ref, held, 1)
    s.update(c=c, pool=pool, table=ints(table), length=ints(length), ref=ints(ref))
    if own:
        from paper_2508_14544_gb300 import KVCache
        s["cache"] = KVCache.wrap(s["pool"], s["table"], s["length"], s["ref"])
    return s


# ---- plain forms: elementary operations on the whole batch, in 32 bits ---------------------------------------------------------

def _pages_of(s, tokens):
    P = s["pool"].shape[4]
    return torch.div(tokens + (P - 1), P, rounding_mode="floor")


def _plain_attend(s):
    pool, q, P = s["pool"], s["q"], s["pool"].shape[4]
    H, D, dev = pool.shape[3], pool.shape[5], q.device
    seqs, cu, n = s["seqs"].long(), s["cu_q"].long(), s["seqs"].numel()
    G, mq = q.shape[1] // H, s["max_q"]
    length, nq = s["length"][seqs].long(), cu[1:] - cu[:-1]
    pos = torch.arange(s["max_len"], device=dev)
    page = s["table"][seqs][:, pos // P].long().clamp(min=0)
    off = (pos % P)[None].expand_as(page)
    at = (cu[:-1, None] + torch.arange(mq, device=dev)[None]).clamp(max=max(s["n_q"] - 1, 0))
    x = q[at].float().view(n, mq, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, mq * G, D)
    k = pool[page, 0, 0, :, off].float().permute(0, 2, 3, 1)
    sc = torch.matmul(x, k) * D ** -0.5
    del k
    last = length[:, None] - nq[:, None] + torch.arange(mq, device=dev)[None]
    hid = pos[None, None] > last[:, :, None]
    sc = sc.view(n, H, mq, G, -1).masked_fill_(hid[:, None, :, None], float("-inf"))
    m = sc.amax(-1, keepdim=True).clamp(min=-3e38)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = pool[page, 0, 1, :, off].float().permute(0, 2, 1, 3)
    o = torch.matmul(p.view(n, H, mq * G, -1), v).view(n, H, mq, G, D) / total.clamp(min=1e-38)
    lse = (m + total.log()).squeeze(-1)
    t = torch.arange(s["n_q"], device=dev)
    i = torch.searchsorted(cu[1:], t, right=True)
    j = t - cu[i]
    return {"out": o[i, :, j].reshape(-1, H * G, D).to(q.dtype), "lse": lse[i, :, j].reshape(-1, H * G)}


def _plain_extend(s, seqs, cu, total, copy_from=None):
    """Pages for `cu`'s new tokens; a shared page that gets some of them is copied first.  With `copy_from`, all of that sequence's pages."""
    pool, table, length, ref, P = s["pool"], s["table"], s["length"], s["ref"], s["pool"].shape[4]
    seqs, cu = seqs.long(), cu.long()
    n, dev = seqs.numel(), seqs.device
    L, new = length[seqs].long(), cu[1:] - cu[:-1]
    have = _pages_of(s, L)
    last = table[seqs, (have - 1).clamp(min=0)].long().clamp(min=0)
    cow = ((new > 0) & (L % P != 0) & (ref[last] > 1)).long()
    need = _pages_of(s, L + new) - have + cow
    i = torch.repeat_interleave(torch.arange(n, device=dev), need)
    nth = torch.arange(i.numel(), device=dev)
    base = need.cumsum(0) - need
    at = have[i] - cow[i] + nth - base[i]
    page = (ref == 0).nonzero()[: i.numel(), 0]
    if copy_from is not None:
        pool[page] = pool[table[copy_from.long()[i], at].long()]
    hit = cow.bool()
    old = last[hit]
    pool[page[base[hit]]] = pool[old]
    ref.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    table[seqs[i], at] = page.int()
    ref[page] = 1
    length[seqs] = (L + new).int()
    i = torch.repeat_interleave(torch.arange(n, device=dev), new)
    pos = L[i] + torch.arange(total, device=dev) - cu[i]
    return table[seqs[i], pos // P].long() * P + pos % P


def _plain_write(s, slots):
    P = s["pool"].shape[4]
    s["pool"][slots // P, 0, 0, :, slots % P] = s["k"]
    s["pool"][slots // P, 0, 1, :, slots % P] = s["v"]


def _plain_free(s, seqs, keep=None):
    table, length, ref, seqs = s["table"], s["length"], s["ref"], seqs.long()
    keep = torch.zeros_like(length[seqs]) if keep is None else torch.minimum(keep, length[seqs])
    rows = table[seqs]
    gone = (rows >= 0) & (torch.arange(rows.shape[1], device=rows.device)[None] >= _pages_of(s, keep)[:, None])
    pages = rows[gone].long()
    ref.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    table[seqs] = rows.masked_fill(gone, -1)
    length[seqs] = keep


def _plain_fork(s, src, dst):
    table, ref, src, dst = s["table"], s["ref"], src.long(), dst.long()
    rows = table[src]
    pages = rows[rows >= 0].long()
    ref.index_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
    table[dst] = rows
    s["length"][dst] = s["length"][src]


def _plain_compact(s):
    pool, table, ref = s["pool"], s["table"], s["ref"]
    live = ref > 0
    n = int(live.sum())
    holes, movers = (~live[:n]).nonzero()[:, 0], live[n:].nonzero()[:, 0] + n
    to = torch.arange(ref.numel(), device=ref.device, dtype=torch.int32).masked_fill(~live, -1)
    to[movers] = holes.int()
    pool[holes] = pool[movers]
    ref[holes] = ref[movers]
    ref[movers] = 0
    table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)], table))
    return to


def _pages(s, extend, write, free, fork, copy, compact):
    """One pass: the step's calls, and those that bring the lengths back to where they were."""
    kind, out = s["c"]["kind"], {}
    if kind == "step":
        out["slots"] = extend(s["seqs"], s["cu_new"], s["total"])
        write(out["slots"])
        free(s["seqs"], s["keep"])
    elif kind == "admit":
        out["slots"] = extend(s["seqs"], s["cu_new"], s["total"])
        write(out["slots"])
        free(s["seqs"], None)
    elif kind == "fork":
        fork(s["src"], s["seqs"])
        out["slots"] = extend(s["seqs"], s["cu_new"], s["total"])
        write(out["slots"])
        free(s["seqs"], None)
    elif kind == "copy":
        copy(s["seqs"], s["dst"])
        free(s["dst"], None)
    else:
        seqs, cu, total = s["parts"][s["turn"] % len(s["parts"])]
        s["turn"] += 1
        free(seqs, None)
        out["to"] = compact()
        out["slots"] = extend(seqs, cu, total)
    # what was moved is compared bit by bit
    return dict(out, pool=s["pool"].view(torch.int16), table=s["table"], length=s["length"], ref=s["ref"])


def run(s):
    if not own:
        if s["c"]["op"] == "attend":
            return _plain_attend(s)

        def copy(src, dst):
            cu = torch.nn.functional.pad(s["length"][src.long()].cumsum(0), (1, 0))
            _plain_extend(s, dst, cu, int(cu[-1]), copy_from=src)
        return _pages(s, lambda a, b, t: _plain_extend(s, a, b, t), lambda x: _plain_write(s, x), lambda a, k: _plain_free(s, a, k),
                      lambda a, b: _plain_fork(s, a, b), copy, lambda: _plain_compact(s))
    kv = s["cache"]
    if s["c"]["op"] == "attend":
        plan = kv.plan(s["seqs"], s["cu_q"], s["n_q"], heads=s["q"].shape[1], cu_group=s["cu_group"])
        out, lse = kv.attend(s["q"], plan)
        return {"out": out, "lse": lse}
    return _pages(s, kv.extend, lambda x: kv.write(x, s["k"], s["v"]), kv.free, kv.fork, kv.copy, kv.compact)


def exact(case, seed):
    """Attention from its definition in 64 bits, a sequence at a time; the pages' outputs are whole numbers."""
    if case["op"] != "attend":
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    P, (_, _, _, H, _, D) = case["page"], s["pool"].shape
    table, cu = s["table"].cpu().numpy(), s["cu_q"].tolist()
    out, lse = [], []
    for i, size in enumerate(s["length"].tolist()):
        rows = torch.from_numpy(table[i, : -(-size // P)].astype(np.int64)).cuda()
        kv = s["pool"][rows, 0].permute(1, 2, 0, 3, 4).reshape(2, H, -1, D)[:, :, :size].double()  # [2, H, size, D]
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
