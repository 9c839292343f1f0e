"""The operators of the 4-bit cache as a program uses them: together, on streams and in graphs, in large pools, in a replay."""
import math

import numpy as np
import pytest

from tests.kv_4bit_reference import held
from tests.test_gpu_kv_4bit import Pool, attend, check, f64, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [1, 4, 32])
@pytest.mark.parametrize("queries,lens", [
    ([20, 0, 0, 3, 0, 17] + [0, 1] * 3 + [0] * 34, [300, 5, 0, 3, 70, 30] + [200] * 40),   # as many tokens as entries at most, unevenly
    ([0] * 29 + [30], [9] * 29 + [10]),                                       # rows of the first tokens see nothing
    ([40] + [0] * 60, [35] + [1] * 60),
    ([33] + [0] * 40, [1500] + [0] * 40),
])
def test_more_rows_than_a_pass_has(queries, lens, group):
    c = Pool(lens, kv_heads=2, dim=64, seed=group)
    check(c, queries, *attend(c, queries, group))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [32, 96, 128])
def test_rows_around_the_sizes_of_items(dim, dtype):
    rows = [1, 7, 8, 9, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 287, 288, 289, 512]
    c = Pool([t + 90 for t in rows], kv_heads=2, dim=dim, dtype=dtype, seed=dim)
    check(c, rows, *attend(c, rows, 1))


@pytest.mark.parametrize("sequences,tokens", [(12, 40), (30, 1)])  # rows of heavy, of light items
def test_long_stretches_in_several_segments(sequences, tokens):
    """More tiles for a block than a segment has: what it has left in the workspace is added to."""
    import torch
    n = 256 * 128 * 2 + 77
    c = Pool([n] * sequences, kv_heads=8, dim=32, page=128, make=lambda m: torch.randn(m, 8, 32, device="cuda"))
    q, out, lse = attend(c, [tokens] * sequences, 1)
    for i in (0, sequences - 1):
        k, v = (x.transpose(1, 0, 2) for x in c.want(i))
        for t in {0, tokens - 1}:
            see, row = n - tokens + t + 1, tokens * i + t
            s = np.einsum("hd,hnd->hn", f64(q[row]), k[:, :see]) * 32 ** -0.5
            w = np.exp(s - s.max(-1, keepdims=True))
            want = np.einsum("hn,hnd->hd", w, v[:, :see]) / w.sum(-1, keepdims=True)
            mag = np.einsum("hn,hnd->hd", w, np.abs(v[:, :see])) / w.sum(-1, keepdims=True)
            # as for shorter ones; products' sums are cut off after every 16 keys, over 256 tiles at most: 2^-13 of them
            assert (np.abs(f64(out[row]) - want) <= 2.0 ** -8 * 1.05 * (mag + np.abs(want)) + 2.0 ** -11 * mag).all()
            assert (np.abs(f64(lse[row]) - (s.max(-1) + np.log(w.sum(-1)))) <= 2e-4).all()


def test_a_pool_of_more_than_four_gigabytes():
    import torch

    from paper_2508_14544_gb300 import KVCache
    P, H, D = 128, 8, 128
    n_pages = (5 << 30) // (2 * H * P * 80)
    kv = KVCache(n_pages, P, H, D, 2, 8, bits=4)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages = [n_pages - 1, 0, n_pages - 3]
    kv.table[0, :3] = ints(pages)
    kv.length[0] = n = 300
    k, v = (torch.randn(n, H, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(n, device="cuda")
    kv.write(torch.tensor(pages, device="cuda")[pos // P] * P + pos % P, k, v)
    rk, rv = kv.read(ints([0]), ints([0, n]), n)
    same(rk, held(f64(k), "bfloat16"))
    same(rv, held(f64(v), "bfloat16"))
    q = torch.randn(1, 64, D, device="cuda").to(torch.bfloat16)
    for rows in (64, 320):  # light and heavy items
        q = torch.randn(1, rows, D, device="cuda").to(torch.bfloat16)
        out, _ = kv.attend(q, kv.plan(ints([0]), ints([0, 1]), 1, heads=rows))
        s = torch.einsum("hgd,nhd->hgn", q[0].double().view(H, -1, D), rk.double()) * D ** -0.5
        want = torch.einsum("hgn,nhd->hgd", s.softmax(-1), rv.double()).reshape(rows, D)
        assert (out[0].double() - want).abs().max() < 0.02
    kv.check()


def test_two_caches_on_two_streams():
    import torch
    cs = [Pool([500, 90], dim=128, seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for c, st in zip(cs, streams):
            with torch.cuda.stream(st):
                got.append((c, attend(c, [1, 2], 8), c.kv.read(c.ints([1]), c.ints([0, 90]), 90)))
    torch.cuda.synchronize()
    for c, (q, out, lse), (k, v) in got:
        check(c, [1, 2], q, out, lse)
        same(k, c.want(1)[0])
        same(v, c.want(1)[1])


def test_graphs_of_two_plans():
    """Two captured steps of one cache, each with its own plan and workspace, replayed in turn."""
    import torch
    c = Pool([700, 300, 5], dim=64)
    seqs, cu = c.ints([0, 1, 2]), c.ints([0, 1, 2, 3])
    qs = [torch.randn(3, h, 64, device="cuda").to(c.dt) for h in (8, 64)]
    side = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for q in qs:
            c.kv.attend(q, c.kv.plan(seqs, cu, 3, heads=q.shape[1]))
    torch.cuda.synchronize()
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(c.kv.attend(q, c.kv.plan(seqs, cu, 3, heads=q.shape[1])))
        graphs.append(g)
    for turn in range(2):
        for q, g in zip(qs, graphs):
            q.normal_()
            g.replay()
        torch.cuda.synchronize()
        for q, (out, lse) in zip(qs, outs):
            check(c, [1, 1, 1], q, out, lse)


def test_prompts_and_steps_of_a_batch():
    """Prompts admitted, attended to, read back; then tokens one by one, with a fork of the longest; every step against 64 bits."""
    import torch

    from paper_2508_14544_gb300 import KVCache
    H, G, D, dt = 2, 4, 80, torch.float16
    kv = KVCache(40, 16, H, D, 4, 12, dtype=dt, bits=4)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator("cuda").manual_seed(0)
    have = {}

    def step(seqs, counts):
        n = sum(counts)
        cu = ints(np.cumsum([0, *counts]))
        slots = kv.extend(ints(seqs), cu, n)
        k, v = (torch.randn(n, H, D, generator=g, device="cuda").to(dt) for _ in range(2))
        q = torch.randn(n, H * G, D, generator=g, device="cuda").to(dt)
        kv.write(slots, k, v)
        out, lse = kv.attend(q, kv.plan(ints(seqs), cu, n, heads=H * G))
        a = 0
        for s, c in zip(seqs, counts):
            x = torch.stack([k[a: a + c], v[a: a + c]])
            have[s] = torch.cat([have[s], x], 1) if s in have else x
            kk, vv = (held(f64(y), "float16") for y in have[s])
            size = kk.shape[0]
            for t in range(c):
                see = size - c + t + 1
                sc = np.einsum("hgd,nhd->hgn", f64(q[a + t]).reshape(H, G, D), kk[:see]) * D ** -0.5
                w = np.exp(sc - sc.max(-1, keepdims=True))
                z = w.sum(-1)
                want = (np.einsum("hgn,nhd->hgd", w, vv[:see]) / z[..., None]).reshape(H * G, D)
                mag = (np.einsum("hgn,nhd->hgd", w, np.abs(vv[:see])) / z[..., None]).reshape(H * G, D)
                assert (np.abs(f64(out[a + t]) - want) <= 2.1 * 2.0 ** -11 * mag + 2.0 ** -12 * mag + see * 2.0 ** -23).all()
                assert (np.abs(f64(lse[a + t]) - (sc.max(-1) + np.log(z)).reshape(-1)) <= 1e-4).all()
            a += c

    step([0, 1, 2], [50, 7, 33])
    kv.fork(ints([0]), ints([3]))
    have[3] = have[0]
    for _ in range(18):
        step([3, 0, 1, 2], [1, 1, 1, 1])
    lens = [have[s].shape[1] for s in range(4)]
    k, v = kv.read(ints([2, 3]), ints([0, lens[2], lens[2] + lens[3]]), lens[2] + lens[3])
    same(k[: lens[2]], held(f64(have[2][0]), "float16"))
    same(v[lens[2]:], held(f64(have[3][1]), "float16"))
    kv.check()


def test_replay_of_a_schedule():
    from paper_2508_14544_gb300 import replay
    from paper_2508_14544_gb300 import workloads as W
    w = W.make_workload("c1", [0])
    r = replay.run(w, 0, "A_max", layers=2, kv_heads=2, group=4, head_dim=64, bits=4, prefix=40)
    assert r["bits"] == 4 and r["steps"] > 0 and math.isfinite(r["us_per_step"])


def test_pages_and_tables_of_bytes():
    """fork, copy, extend and compact move a 4-bit cache's pages as bytes: what is read afterwards is what was."""
    import torch
    c = Pool([40, 100], dim=96, page=32)
    kv, ints = c.kv, c.ints
    before = kv.read(ints([1]), ints([0, 100]), 100)
    kv.free(ints([0]))
    kv.compact()
    after = kv.read(ints([1]), ints([0, 100]), 100)
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    kv.check()
