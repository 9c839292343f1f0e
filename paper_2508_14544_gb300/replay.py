"""Run the key/value side of a simulated schedule on the GPU and fit the batch-time model to it.

  python -m paper_2508_14544_gb300.replay [--workload c1] [--instance 0] [--policy A_max] [--layers 4] [--kv-heads 8]
                                          [--group 8] [--head-dim 128] [--page 16] [--bits 16] [--prefix 0] [--steps N]

One instance is simulated under a policy that cancels nothing (A_max, H-SF, A_r), whose completions give every
request's start: C_i - o_i.  Its batches are then run on a ``KVCache``, step by step: a request that starts gets
pages for its prompt and first token, the others one token each; keys and values are written and attended to in every layer; a
request that completes gives its pages back.  With ``--prefix`` all requests are forked from one sequence of that many
tokens, which is read once for the batch; with ``--bits 4`` the cache holds keys and values in 4 bits.  Values are random: what is measured is the time of the memory that the
schedulers count, not a model.

The steps' times are fitted to Section 6's linear batch-time model, c0 + c1 |B| + c2 (KV tokens) + c3 (prompt tokens
started), and ``Simulator.batch_time`` gives the schedule's total latency and makespan with these coefficients (in
microseconds).  Prints one JSON line.
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from . import POLICIES, KVCache, Simulator
from . import workloads as W

WITHOUT_CANCELLATIONS = ("A_max", "H-SF", "A_r")


def batches(start, completion) -> list:
    """Per processed step: (requests that start, requests that go on, requests that complete), as index arrays."""
    start, completion = np.asarray(start), np.asarray(completion)
    out = []
    for t in np.unique(np.concatenate([np.arange(a, b) for a, b in zip(start, completion)] or [np.zeros(0, int)])):
        on = (start <= t) & (t < completion)
        out.append((np.flatnonzero(on & (start == t)), np.flatnonzero(on & (start < t)), np.flatnonzero(completion == t + 1)))
    return out


def run(w, row: int = 0, policy: str = "A_max", layers: int = 4, kv_heads: int = 8, group: int = 8, head_dim: int = 128,
        page: int = 16, prefix: int = 0, max_steps: int | None = None, bits: int = 16) -> dict:
    """Replay instance ``row`` of a Workload; see the module."""
    import torch
    if policy not in WITHOUT_CANCELLATIONS:
        raise ValueError(f"policy must be one of {WITHOUT_CANCELLATIONS}: others' completions do not give their schedule")
    w = w.subset([row])
    inst = w.instance(0)
    s, o = np.asarray(inst["s"]), np.asarray(inst["o"])
    with Simulator(POLICIES[policy], w.M, 1, record_completions=1, batch_time=1) as sim:
        sim.load_workload(w)
        res = sim.run()[0]
        if res["status"] != 0:
            raise RuntimeError(f"the instance failed with status {int(res['status'])}")
        completion = sim.completions(w.n_total)
        steps = batches(completion - o, completion)
        most = max(len(a) + len(b) for a, b, _ in steps)
        longest = prefix + int((s + o).max())
        # pages: each sequence's last one may be nearly empty, and its first tokens may share the prefix's last one
        n_pages = -(-prefix // page) + w.M // page + 2 * most + 2
        kv = KVCache(n_pages, page, kv_heads, head_dim, most + 1, -(-longest // page) + 1, n_layers=layers, bits=bits)
        ints = lambda x: torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")  # noqa: E731

        def values(n, heads):
            return torch.randn(n, heads, head_dim, device="cuda", dtype=torch.bfloat16)

        root = ints([most])
        if prefix:
            slots = kv.extend(root, ints([0, prefix]), prefix)
            for layer in range(layers):
                kv.write(slots, values(prefix, kv_heads), values(prefix, kv_heads), layer=layer)
        seq_of, free = {}, list(range(most))[::-1]
        length = np.zeros(len(s), np.int64)
        rows, times, peak = [], [], 0
        for new, old, done in steps[:max_steps]:
            for i in new:
                seq_of[int(i)] = free.pop()
            members = np.concatenate([new, old])
            tokens = np.concatenate([s[new] + 1, np.ones(len(old), s.dtype)])
            length[members] += tokens
            n_q = int(tokens.sum())
            seqs, cu = ints([seq_of[int(i)] for i in members]), ints(np.concatenate([[0], np.cumsum(tokens)]))
            starting = ints([seq_of[int(i)] for i in new])
            ending = ints([seq_of[int(i)] for i in done])
            whole = ints([0, len(members)])
            k, v, q = values(n_q, kv_heads), values(n_q, kv_heads), values(n_q, kv_heads * group)
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            if prefix and len(new):
                kv.fork(root.expand(len(new)).contiguous(), starting)
            slots = kv.extend(seqs, cu, n_q)
            plan = kv.plan(seqs, cu, n_q, heads=kv_heads * group, cu_group=whole if prefix else None)
            for layer in range(layers):
                kv.write(slots, k, v, layer=layer)
                out, _ = kv.attend(q, plan, layer=layer)
            kv.free(ending)
            b.record()
            mem = int(length[members].sum())
            peak = max(peak, mem)
            rows.append((1.0, float(len(members)), float(mem), float(s[new].sum())))
            times.append((a, b))
            for i in done:
                free.append(seq_of.pop(int(i)))
        kv.check()
        ms = np.array([a.elapsed_time(b) for a, b in times])
        skip = min(3, len(ms) - 1)  # the first steps include what is set up once
        fit, *_ = np.linalg.lstsq(np.array(rows)[skip:], ms[skip:] * 1e3, rcond=None)
        coef = [float(x) for x in fit] + [0.0]
        total, makespan = sim.batch_time(coef)[0]
    if max_steps is None:
        assert peak == int(res["peak_memory"]) and not kv.length[:most].any()
    return {"workload": w.name, "policy": policy, "requests": len(s), "M": int(w.M), "steps": len(ms), "peak_tokens": peak,
            "layers": layers, "kv_heads": kv_heads, "q_heads": kv_heads * group, "head_dim": head_dim, "bits": bits, "prefix": prefix,
            "us_per_step": float(ms[skip:].mean() * 1e3), "coef_us": coef, "total_latency_us": float(total),
            "makespan_us": float(makespan)}


def main(argv=None) -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="c1", choices=sorted(W.WORKLOADS))
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--policy", default="A_max", choices=WITHOUT_CANCELLATIONS)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--group", type=int, default=8, help="query heads per kv head")
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--bits", type=int, default=16, choices=(16, 4), help="of a cached value")
    ap.add_argument("--prefix", type=int, default=0, help="tokens of a prompt that all requests share")
    ap.add_argument("--steps", type=int, default=None, help="only the first N batches")
    args = ap.parse_args(argv)
    print(json.dumps(run(W.make_workload(args.workload, [args.instance]), 0, args.policy, args.layers, args.kv_heads, args.group,
                         args.head_dim, args.page, args.prefix, args.steps, args.bits)))


if __name__ == "__main__":
    main()
