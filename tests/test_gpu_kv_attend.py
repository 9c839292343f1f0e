"""Attention over the paged cache against 64 bits, at the lengths, heads, pages and masks where it can go wrong."""
import math

import numpy as np
import pytest

from tests.kv_reference import attention

pytestmark = pytest.mark.gpu
ROUND = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}  # unit roundoff


class Case:
    """Sequences of the lengths given, on pages in random order, the rest of the pool filled with `rest`."""

    def __init__(self, lens, queries, kv_heads=2, group=4, dim=64, page=16, dtype="bfloat16", layers=1, layer=0, groups=None, prefix=0,
                 rest=math.nan, seed=0, spread=1.0):
        import torch

        from paper_2508_14544_gb300 import KVCache
        rng = np.random.default_rng(seed)
        self.torch, self.dtype, self.layer, self.group = torch, dtype, layer, group
        dt, P = getattr(torch, dtype), page
        self.lens, self.queries = list(lens), list(queries)
        shared = prefix // P
        most = max([-(-x // P) for x in lens] + [1]) + 1
        n_pages = sum(-(-x // P) for x in lens) + shared * (len(groups) if groups else 0) + 3
        order = rng.permutation(n_pages).tolist()
        table = np.full((len(lens) + 1, most), -1, np.int32)
        bounds = [0, *np.cumsum(groups).tolist()] if groups else []
        for a, b in zip(bounds, bounds[1:]):
            first = [order.pop() for _ in range(shared)]
            for i in range(a, b):
                k = min(shared, lens[i] // P)
                table[i, :k] = first[:k]
        for i, x in enumerate(lens):
            for j in range(-(-x // P)):
                if table[i, j] < 0:
                    table[i, j] = order.pop()
        g = torch.Generator("cuda").manual_seed(seed)
        pool = torch.full((n_pages, layers, 2, kv_heads, P, dim), rest, dtype=dt, device="cuda")
        for i, x in enumerate(lens):
            for j in range(-(-x // P)):
                n = min(P, x - j * P)
                pool[int(table[i, j]), :, :, :, :n] = torch.randn(layers, 2, kv_heads, n, dim, generator=g, device="cuda").to(dt)
        length = np.array([*lens, 0], np.int32)
        ref = np.zeros(n_pages, np.int32)
        np.add.at(ref, table[table >= 0], 1)
        ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        self.ints = ints
        self.kv = KVCache.wrap(pool, ints(table), ints(length), ints(ref))
        self.seqs, self.cu = ints(range(len(lens))), ints([0, *np.cumsum(queries)])
        self.n_q = int(sum(queries))
        self.q = (torch.randn(self.n_q, kv_heads * group, dim, generator=g, device="cuda") * spread).to(dt)
        self.table, self.bounds = table, ints(bounds) if bounds else None

    def run(self, grouped=True, q=None, scale=None, **more):
        plan = self.kv.plan(self.seqs, self.cu, self.n_q, heads=self.q.shape[1], cu_group=self.bounds if grouped else None)
        return self.kv.attend(self.q if q is None else q, plan, layer=self.layer, scale=scale, **more)

    def check(self, out, lse, scale=None):
        torch, dim = self.torch, self.q.shape[2]
        scale = dim ** -0.5 if scale is None else scale
        u, at = ROUND[self.dtype], 0
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        pool = self.kv.pool[:, self.layer]
        for i, (n, t) in enumerate(zip(self.lens, self.queries)):
            rows = torch.from_numpy(self.table[i][: -(-n // self.kv.pool.shape[4])].astype(np.int64)).cuda()
            kv = pool[rows].double().cpu().numpy().transpose(1, 2, 0, 3, 4).reshape(2, pool.shape[2], -1, dim)[:, :, :n]
            want, wl, mag = attention(self.q[at: at + t].double().cpu().numpy(), kv[0], kv[1], scale)
            # P is rounded to 16 bits (and, in float16, below 2^-24 to multiples of that), the result again; sums and
            # exponentials in 32 bits: 2^-12 of the magnitudes covers products of up to 10^4 terms
            floor = n * 2.0 ** -25 * (np.abs(kv[1]).max() if n else 0) if self.dtype == "float16" else 0
            tol = 1.05 * u * (mag + np.abs(want)) + 2.0 ** -12 * mag + floor
            got = out[at: at + t]
            bad = ~(np.abs(got - want) <= tol)
            assert not bad.any(), (i, n, t, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])
            gl = lse[at: at + t]
            none = np.isneginf(wl)
            assert np.array_equal(np.isneginf(gl), none)
            assert np.all(np.abs(gl[~none] - wl[~none]) <= 2e-5 * np.maximum(1, np.abs(wl[~none]))), (i, n, t)
            at += t
        self.kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (80, 64), (8, 128), (72, 16), (128, 128)])
def test_single_tokens_over_many_lengths(dtype, dim, page):
    lens = [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 130, 200, 255, 256, 257, 300, 511, 700]
    c = Case(lens, [1] * len(lens), dim=dim, page=page, dtype=dtype, seed=dim + page)
    c.check(*c.run())


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (1, 7), (2, 16), (3, 33), (1, 64), (2, 65), (1, 128), (1, 129), (1, 300), (5, 3)])
def test_head_layouts(kv_heads, group):
    lens = [1, 40, 129, 300]
    c = Case(lens, [1] * 4, kv_heads=kv_heads, group=group, seed=group)
    c.check(*c.run())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,queries,group", [
    ([5, 1, 130, 300], [5, 1, 130, 300], 1),        # whole prompts
    ([77, 300, 128], [20, 33, 128], 4),             # 80, 132, 512 rows
    ([500, 400], [37, 16], 8),                      # light remainders after heavy items
    ([64, 65, 200], [3, 0, 5], 5),                  # an entry without queries
    ([260], [257], 3),
])
def test_many_queries_see_the_keys_up_to_their_own(lens, queries, group, dim):
    c = Case(lens, queries, group=group, dim=dim, seed=len(lens))
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4])
def test_rows_around_the_sizes_of_items(group, dim, dtype):
    """Up to 32, 128 and 256 rows and just over, whole items and what is left after them, side by side."""
    rows = [31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 287, 288, 289, 385, 512]
    queries = [-(-r // group) for r in rows]
    c = Case([t + 90 for t in queries], queries, group=group, dim=dim, dtype=dtype, kv_heads=3, seed=group)
    c.check(*c.run())


@pytest.mark.parametrize("groups", [None, [1, 399, 0, 500, 300]])
def test_more_entries_than_the_plan_keeps_on_chip(groups):
    rng = np.random.default_rng(5)
    n, prefix = 1200, 160 if groups else 0
    lens = (prefix + rng.integers(0, 70, n)).tolist()
    queries = [int(rng.integers(0, min(x, 3) + 1)) for x in lens]
    c = Case(lens, queries, kv_heads=1, group=4, groups=groups, prefix=prefix, seed=9)
    c.check(*c.run())


@pytest.mark.parametrize("group", [1, 4, 32])
@pytest.mark.parametrize("queries,lens", [
    ([20, 0, 0, 3, 0, 17] + [0, 1] * 3 + [0] * 34, [300, 5, 0, 3, 70, 30] + [200] * 40),   # as many tokens as entries at most, unevenly
    ([0] * 29 + [30], [9] * 29 + [10]),                                       # rows of the first tokens see nothing
    ([40] + [0] * 60, [35] + [1] * 60),
    ([33] + [0] * 40, [1500] + [0] * 40),
])
def test_no_more_tokens_than_entries(queries, lens, group):
    assert sum(queries) <= len(queries)
    c = Case(lens, queries, group=group, dim=128 if group == 4 else 72, seed=group)
    c.check(*c.run())


def test_plans_that_are_gone_leave_their_room_to_the_next():
    a, b = Case([900, 40], [1, 1], seed=1), Case([300] * 30, [3] * 30, seed=2)
    for c in (a, b, a, b):
        for _ in range(3):
            c.check(*c.run())
    torch = a.torch
    want = a.run()
    plan = a.kv.plan(a.seqs, a.cu, a.n_q, heads=a.q.shape[1])
    other = a.kv.plan(a.seqs, a.cu, a.n_q, heads=a.q.shape[1])
    assert plan._buffer.data_ptr() != other._buffer.data_ptr()
    assert torch.equal(a.kv.attend(a.q, plan)[0], want[0]) and torch.equal(a.kv.attend(a.q, other)[0], want[0])
    room = other._buffer.data_ptr()
    del other
    third = a.kv.plan(a.seqs, a.cu, a.n_q, heads=a.q.shape[1])
    assert third._buffer.data_ptr() == room != plan._buffer.data_ptr()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # read on another stream: not the next one's
        out = a.kv.attend(a.q, third)[0]
    torch.cuda.current_stream().wait_stream(side)
    del third
    assert a.kv._spare == [] and torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = a.kv.attend(a.q, plan)
        own = a.run()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(own[0], want[0]) and torch.equal(captured[0], want[0])
    del plan  # the graph may be replayed: its plan's room is no other's
    assert a.kv._spare == []
    a.kv.check()


def test_rows_that_see_nothing():
    """More queries than tokens, and sequences without any: zeros and -infinity."""
    for lens, queries in (([0, 3, 0], [2, 5, 1]), ([0], [1]), ([2], [300])):
        c = Case(lens, queries, rest=math.inf)
        out, lse = c.run()
        c.check(out, lse)
        assert not out[:1].any() and math.isinf(lse[0, 0].item())


@pytest.mark.parametrize("rest", [math.nan, math.inf, -math.inf, 6e4])
@pytest.mark.parametrize("group", [2, 20, 40, 100, 200])
def test_what_lies_past_the_end_is_not_used(rest, group):
    c = Case([1, 5, 33, 100, 129, 250], [1] * 6, group=group, rest=rest, dtype="float16", page=64)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens,queries,group,dim", [([70, 200], [6, 5], 3, 64), ([300, 65], [30, 40], 2, 80), ([500], [200], 4, 128), ([5000], [7], 2, 128)])
def test_keys_that_a_query_does_not_see_yet(lens, queries, group, dim, bad, dtype):
    """The newest tokens' keys and values are infinite or not a number: queries before them are as without them."""
    c = Case(lens, queries, group=group, dim=dim, dtype=dtype, kv_heads=1, seed=7)
    torch, P, at = c.torch, c.kv.pool.shape[4], 0
    out, lse = c.run()
    c.check(out, lse)
    keep = torch.zeros(c.n_q, dtype=torch.bool, device="cuda")
    for i, (n, t) in enumerate(zip(lens, queries)):
        new = t // 3 + 1  # so many of the last tokens
        for x in range(n - new, n):
            page = int(c.table[i, x // P])
            c.kv.pool[page, :, 1, :, x % P, x % dim] = bad  # one value of each; of the very last also the keys
            if x == n - 1:
                c.kv.pool[page, :, 0, :, x % P] = bad
        keep[at: at + t - new] = True
        at += t
    got, glse = c.run()
    u = ROUND[dtype]
    assert torch.isfinite(got[keep]).all() and (glse[keep] - lse[keep]).abs().max() <= 1e-5
    # the probabilities of these rows may have been rounded in one run and not in the other
    assert ((got[keep].float() - out[keep].float()).abs() <= 2.5 * u * out[keep].float().abs().clamp(min=0.5) + 4 * u).all()
    assert not torch.isfinite(got[~keep]).all(dim=-1).all(dim=-1).any()


@pytest.mark.parametrize("dtype,dim,page,group", [("bfloat16", 128, 16, 8), ("float16", 80, 32, 5), ("bfloat16", 64, 64, 1), ("float16", 128, 128, 3)])
def test_shared_prefixes(dtype, dim, page, group):
    groups, prefix = [40, 1, 9, 3], 1500
    rng = np.random.default_rng(page)
    lens = [prefix + int(rng.integers(1, 200)) for _ in range(53)]
    c = Case(lens, [1] * 53, dim=dim, page=page, group=group, dtype=dtype, groups=groups, prefix=prefix, seed=page)
    out, lse = c.run()
    c.check(out, lse)
    plain, plain_lse = c.run(grouped=False)
    c.check(plain, plain_lse)
    assert (out.float() - plain.float()).abs().max() < 0.02 and (lse - plain_lse).abs().max() < 1e-4


def test_shared_prefixes_at_their_edges():
    """Entries that end with the prefix, inside it, before it; with several queries; without any."""
    P, prefix = 16, 640
    lens = [640, 641, 656, 700, 640, 650, 645, 800]
    c = Case(lens, [1, 1, 3, 60, 1, 11, 0, 2], groups=[8], prefix=prefix, page=P)
    c.check(*c.run())
    c = Case([640, 640, 640, 640] * 8, [1] * 32, groups=[32], prefix=prefix, page=P)  # forks that have nothing of their own
    c.check(*c.run())
    c = Case([640, 30, 700, 640], [1, 1, 1, 1], groups=[4], prefix=prefix, page=P)  # one is shorter than the others' prefix
    c.check(*c.run())
    c = Case([3, 700] + [690] * 30, [7] + [1] * 31, groups=[32], prefix=prefix, page=P)  # one with rows that see nothing
    c.check(*c.run())


def shares(c):
    """Whether a plan of this batch reads prefixes once: entries then have rows to join."""
    plan = c.kv.plan(c.seqs, c.cu, c.n_q, heads=c.q.shape[1], cu_group=c.bounds)
    return int(plan._buffer[:128].view(c.torch.int32)[17]) > 0


@pytest.mark.parametrize("dtype,dim,page,group", [("bfloat16", 128, 16, 8), ("float16", 80, 32, 5), ("bfloat16", 64, 64, 1), ("float16", 128, 128, 3)])
@pytest.mark.parametrize("most", [1, 3, 7])
def test_shared_prefixes_that_are_worth_it(dtype, dim, page, group, most):
    """Groups of one, few and many; prefixes' rows and entries' own ones in light and in heavy items."""
    groups, prefix = [30, 1, 9, 2, 12], 2100
    rng = np.random.default_rng(page + most)
    queries = [int(rng.integers(1, most + 1)) for _ in range(54)]
    lens = [prefix + t - 1 + int(rng.integers(0, 200)) for t in queries]
    c = Case(lens, queries, kv_heads=8, dim=dim, page=page, group=group, dtype=dtype, groups=groups, prefix=prefix, seed=page)
    assert shares(c)
    out, lse = c.run()
    c.check(out, lse)
    again, again_lse = c.run()
    assert c.torch.equal(out, again) and c.torch.equal(lse, again_lse)


@pytest.mark.parametrize("lens,queries", [
    ([1600, 1601, 1616, 1660, 1600, 1610, 1605, 1760] * 5, [1, 1, 3, 20, 1, 11, 0, 2] * 5),  # end with the prefix, inside it, after it; no queries
    ([1600] * 32, [1] * 32),                                                                 # nothing of their own
    ([1650] * 32, [1] * 32),
    ([1660] + [1650] * 30, [33] + [5] * 30),
])
@pytest.mark.parametrize("rest", [float("nan"), float("inf")])
def test_edges_of_prefixes_that_are_worth_it(lens, queries, rest):
    c = Case(lens, queries, kv_heads=8, groups=[len(lens)], prefix=1600, rest=rest)
    assert shares(c)
    c.check(*c.run())


def test_short_prefixes_are_not_shared():
    c = Case([70] * 8, [1] * 8, groups=[8], prefix=64)
    assert not shares(c)
    c.check(*c.run())


def test_a_long_sequence_is_divided():
    c = Case([20011, 3], [1, 1], kv_heads=1, group=8, dim=128, page=128)
    c.check(*c.run())
    c = Case([9001], [40], kv_heads=1, group=8, dim=64, page=32, dtype="float16")
    c.check(*c.run())


def test_scores_far_apart():
    """One key takes all, the running maximum grows many times; a large scale."""
    for spread, scale in ((60.0, None), (3.0, 7.5), (1e-3, None)):
        c = Case([700, 129, 1000], [1, 4, 2], spread=spread, dim=128, dtype="bfloat16", seed=3)
        out, lse = c.run(scale=scale)
        torch = c.torch
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        if spread <= 1:
            c.check(out, lse, scale)
        else:  # scores of hundreds: their own 32-bit rounding moves the exponentials
            want = []
            for i, n in enumerate(c.lens):
                rows = torch.from_numpy(c.table[i][: -(-n // 16)].astype(np.int64)).cuda()
                kv = c.kv.pool[rows, 0].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n].double()
                a, t = sum(c.queries[:i]), c.queries[i]
                s = torch.einsum("thgd,hsd->thgs", c.q[a: a + t].double().unflatten(1, (2, -1)), kv[0]) * (scale or 128 ** -0.5)
                see = torch.arange(n, device="cuda")[None] <= torch.arange(n - t, n, device="cuda")[:, None]
                want.append(s.masked_fill(~see[:, None, None], -math.inf).logsumexp(-1).flatten(1))
            want = torch.cat(want)
            assert ((lse - want).abs() / want.abs().clamp(min=1)).max() < 2e-5


@pytest.mark.parametrize("token,head,offset", [(640, 80, 0), (700, 81, 1), (640, 72, 3)])
def test_strided_and_unaligned_queries_and_strided_results(token, head, offset):
    c = Case([100, 40, 300], [1, 7, 40], dtype="float16")
    torch = c.torch
    raw = torch.empty(c.n_q * 720 + 64, dtype=torch.float16, device="cuda")
    q = raw.as_strided(c.q.shape, (token, head, 1), offset)
    q.copy_(c.q)
    out = torch.full((c.n_q, 11, 96), 5.0, dtype=torch.float16, device="cuda")[:, 2:10, 8:72]
    got, lse = c.run(q=q, out=out)
    assert got.data_ptr() == out.data_ptr()
    c.check(out, lse)


def test_layers_and_the_same_plan():
    c = Case([50, 140], [1, 2], layers=3, layer=2, dim=72)
    c.check(*c.run())
    plan = c.kv.plan(c.seqs, c.cu, c.n_q, heads=c.q.shape[1])
    for layer in (1, 0, 2):
        c.layer = layer
        c.check(*c.kv.attend(c.q, plan, layer=layer))


def test_the_same_result_every_time_and_in_a_graph():
    c = Case([1500, 1400, 1450, 1600], [1, 2, 1, 1], groups=[4], prefix=1300, group=40)
    torch = c.torch
    out, lse = c.run()
    for _ in range(3):
        again, al = c.run()
        assert torch.equal(out, again) and torch.equal(lse, al)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, other[0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = c.run()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, captured[0]) and torch.equal(lse, captured[1])


def test_entries_that_are_refused():
    from paper_2508_14544_gb300 import SimError
    c = Case([50, 60, 70], [1, 1, 1])
    out, lse = c.run()
    c.seqs = c.ints([0, 99, 2])
    got, _ = c.run()
    assert c.torch.equal(got[[0, 2]], out[[0, 2]]) and not got[1].any()
    with pytest.raises(SimError):
        c.kv.check()
    c.seqs, c.cu = c.ints([0, 1, 2]), c.ints([0, 2, 1, 3])  # offsets that decrease
    c.run()
    with pytest.raises(SimError):
        c.kv.check()


def test_no_queries():
    c = Case([50], [0])
    out, lse = c.run()
    assert out.shape[0] == 0 and lse.shape[0] == 0
    c.kv.check()


def test_a_table_with_pages_outside_the_pool_reads_zeros():
    """A page number that no pool has is not followed."""
    c = Case([40], [1], rest=0.0)
    c.kv.table[0, 1] = 1 << 20
    c.kv.table[0, 2] = -5
    out, lse = c.run()
    assert c.torch.isfinite(out).all() and c.torch.isfinite(lse).all()


def test_keys_past_32_bits_of_offset():
    import torch

    from paper_2508_14544_gb300 import KVCache
    kv = KVCache(2100, 128, 8, 128, 1, 4, n_layers=4)
    kv.ref[:2090] = 1
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    slots = kv.extend(ints([0]), ints([0, 400]), 400)
    k, v, q = (torch.randn(n, 8, 128, device="cuda").bfloat16() for n in (400, 400, 1))
    kv.write(slots, k, v, layer=3)
    out, _ = kv.attend(q, kv.plan(ints([0]), ints([0, 1]), 1, heads=8), layer=3)
    w = torch.einsum("thd,shd->ths", q.double(), k.double()).mul(128 ** -0.5).softmax(-1)
    want, mag = torch.einsum("ths,shd->thd", w, v.double()), torch.einsum("ths,shd->thd", w, v.double().abs())
    assert ((out.double() - want).abs() <= 1.05 * 2.0 ** -8 * (mag + want.abs()) + 2.0 ** -12 * mag).all()
    kv.check()
