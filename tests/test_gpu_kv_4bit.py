"""A cache held in 4 bits: what is written against the reference's codes and steps, bit by bit, what is read, and attention over it."""
import math

import numpy as np
import pytest

from tests.kv_4bit_reference import BITS, held, round16
from tests.kv_reference import attention

pytestmark = pytest.mark.gpu
ROUND = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}  # unit roundoff


def f64(x):
    return x.double().cpu().numpy()


def same(got, want):
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = ~((got == want) | np.isnan(want))
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


class Pool:
    """A cache of 4 bits with `lens` tokens in sequences 0, 1, .., on pages in random order, its memory filled with `fill` before."""

    def __init__(self, lens, kv_heads=2, dim=64, page=16, dtype="bfloat16", layers=1, fill=0xff, seed=0, make=None, groups=None, prefix=0):
        import torch

        from paper_2508_14544_gb300 import KVCache
        rng = np.random.default_rng(seed)
        self.torch, self.dtype, self.dt, self.lens, self.dim, self.page, self.heads = torch, dtype, getattr(torch, dtype), list(lens), dim, page, kv_heads
        shared = prefix // page
        most = max([-(-x // page) for x in lens] + [1]) + 1
        n_pages = sum(-(-x // page) for x in lens) + shared * (len(groups) if groups else 0) + 3
        order = rng.permutation(n_pages).tolist()
        self.table = np.full((len(lens) + 1, most), -1, np.int32)
        bounds = [0, *np.cumsum(groups).tolist()] if groups else []
        for a, b in zip(bounds, bounds[1:]):
            first = [order.pop() for _ in range(shared)]
            for i in range(a, b):
                self.table[i, : min(shared, lens[i] // page)] = first[: min(shared, lens[i] // page)]
        for i, x in enumerate(lens):
            for j in range(-(-x // page)):
                if self.table[i, j] < 0:
                    self.table[i, j] = order.pop()
        ref = np.zeros(n_pages, np.int32)
        np.add.at(ref, self.table[self.table >= 0], 1)
        self.kv = KVCache(n_pages, page, kv_heads, dim, len(lens) + 1, most, n_layers=layers, dtype=self.dt, bits=4)
        self.kv.pool.fill_(fill)
        self.kv.table.copy_(self.ints(self.table))
        self.kv.length.copy_(self.ints([*lens, 0]))
        self.kv.ref.copy_(self.ints(ref))
        g = torch.Generator("cuda").manual_seed(seed)
        self.gen = g
        slots = np.unique(np.concatenate([self.slots(i, 0, x) for i, x in enumerate(lens)] + [np.zeros(0, np.int64)]))
        make = make or (lambda n: torch.randn(n, kv_heads, dim, generator=g, device="cuda") * torch.rand(n, 1, 1, generator=g, device="cuda").exp())
        self.k, self.v = (torch.zeros(n_pages * page, kv_heads, dim, dtype=self.dt, device="cuda") for _ in range(2))
        at = torch.from_numpy(slots).cuda()
        self.k[at], self.v[at] = make(len(slots)).to(self.dt), make(len(slots)).to(self.dt)
        self.layer = layers - 1
        self.kv.write(at, self.k[at], self.v[at], layer=self.layer)
        self.bounds = self.ints(bounds) if bounds else None

    def ints(self, x):
        return self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device="cuda")

    def slots(self, i, a, b):
        pos = np.arange(a, b)
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page

    def want(self, i, a=0, b=None):
        """What the cache holds of sequence i's tokens: [2][tokens, heads, dim]."""
        at = self.torch.from_numpy(self.slots(i, a, self.lens[i] if b is None else b)).cuda()
        return held(f64(self.k[at]), self.dtype), held(f64(self.v[at]), self.dtype)


SPECIAL = ["ties", "large", "tiny", "mixed", "equal", "zeros", "integers", "borders", "small lowest"]


def special(kind, torch, dtype):
    def make(n):
        g = torch.Generator("cuda").manual_seed(n)
        x = torch.randn(n, 2, 80, generator=g, device="cuda", dtype=torch.float64)
        most = {"bfloat16": 3.38e38, "float16": 65504.0}[dtype]
        if kind == "ties":  # span 15: step 1, values halfway
            x = torch.round(x * 8).clamp(-15, 15) / 2
            x[..., ::32], x[..., 1::32] = -7.5, 7.5
        elif kind == "large":
            x = (x / 4).clamp(-1, 1) * most
        elif kind == "tiny":
            x = torch.round(x * 9) * 2.0 ** BITS[dtype][1]
        elif kind == "mixed":
            x = x * 2.0 ** torch.randint(-12, 12, x.shape, generator=g, device="cuda")
        elif kind == "equal":
            x = x[..., :1].expand(n, 2, 80).clone()
        elif kind == "zeros":
            x = x * 0
        elif kind == "integers":
            x = torch.round(x * 40)
        elif kind == "borders":  # -lo on or next to a border, values on or next to borders, and others too small for an exact difference
            bits, least, _ = BITS[dtype]
            r = lambda lo, hi, *shape: torch.randint(lo, hi, shape or (n, 2, 1), generator=g, device="cuda").double()  # noqa: E731
            s = r(2 ** (bits - 1), 2 ** bits) * 2.0 ** (r(-4, 5) - bits)
            lo = -(r(0, 15) + 0.5) * s
            lo = torch.from_numpy(round16((lo * (1 + r(-2, 3) * 2.0 ** -bits)).cpu().numpy(), dtype)).cuda()
            x = lo + (r(0, 16, n, 2, 80) + 0.5 * r(0, 2, n, 2, 80)) * s * (1 + r(-1, 2, n, 2, 80) * 2.0 ** -bits)
            tiny = r(-40, 41, n, 2, 80) * 2.0 ** (r(-24, -8, n, 2, 80) if dtype == "float16" else r(-60, -10, n, 2, 80))
            x = torch.where(r(0, 3, n, 2, 80) == 0, tiny, x).clamp(min=lo, max=lo + 15 * s)
            x[..., ::32], x[..., 1::32] = lo, lo + 15 * s
        elif kind == "small lowest":  # lo next to nothing beside the others
            x = torch.round(x.abs() * 64) / 8 + 0.125
            x[..., ::32] = 2.0 ** -torch.randint(8, 24, (n, 2, 3), generator=g, device="cuda").double() * torch.where(x[..., 1::32][..., :3] > 1, 1.0, -1.0)
        return torch.from_numpy(round16(x.cpu().numpy(), dtype)).cuda()
    return make


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page,heads", [(64, 16, 2), (128, 32, 1), (80, 64, 3), (8, 128, 2), (72, 16, 5), (96, 32, 2), (128, 128, 2), (32, 16, 1)])
def test_what_is_written_is_read_back(dim, page, heads, dtype):
    lens = [1, 2, 15, 16, 17, 31, 130, 300]
    c = Pool(lens, kv_heads=heads, dim=dim, page=page, dtype=dtype, layers=2, seed=dim + page)
    cu = np.cumsum([0, *lens])
    k, v = c.kv.read(c.ints(range(len(lens))), c.ints(cu), int(cu[-1]), layer=1)
    for i, x in enumerate(lens):
        wk, wv = c.want(i)
        same(k[cu[i]: cu[i + 1]], wk)
        same(v[cu[i]: cu[i + 1]], wv)
    c.kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("kind", SPECIAL)
def test_values_next_to_borders_and_at_the_ends_of_the_range(kind, dtype):
    import torch
    c = Pool([700], dim=80, dtype=dtype, make=special(kind, torch, dtype))
    k, v = c.kv.read(c.ints([0]), c.ints([0, 700]), 700)
    wk, wv = c.want(0)
    same(k, wk)
    same(v, wv)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_groups_that_are_not_finite(dtype):
    import torch

    def make(n):
        x = torch.randn(n, 2, 80, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        x[::3, 0, 33], x[1::7, 1, 79], x[2::5, 1, 0] = math.inf, math.nan, -math.inf
        return x
    c = Pool([100], dim=80, dtype=dtype, make=make)
    k, v = c.kv.read(c.ints([0]), c.ints([0, 100]), 100)
    wk, wv = c.want(0)
    assert np.isnan(wk).any()
    same(k, wk)
    same(v, wv)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["odd address", "transposed", "one head", "slots"])
def test_sources_of_any_stride_and_alignment(kind, dtype):
    import torch
    c = Pool([64], kv_heads=2, dim=72, dtype=dtype)
    n, dt = 33, c.dt
    x = torch.randn(2, n, 2, 72, device="cuda").to(dt)
    if kind == "odd address":
        big = torch.zeros(2, n * 144 + 1, dtype=dt, device="cuda")
        big[:, 1:] = x.flatten(1)
        k, v = big[0, 1:].view(n, 2, 72), big[1, 1:].view(n, 2, 72)
    elif kind == "transposed":
        y = x.transpose(1, 2).contiguous()
        k, v = y[0].transpose(0, 1), y[1].transpose(0, 1)
    elif kind == "one head":
        x = x[:, :, :1].expand(2, n, 2, 72)
        k, v = x[0], x[1]
    else:
        k, v = x[0], x[1]
    at = torch.randperm(64, device="cuda")[:n]
    slots = torch.from_numpy(c.slots(0, 0, 64)).cuda()[at]
    before = c.kv.read(c.ints([0]), c.ints([0, 64]), 64)
    if kind == "slots":  # none of the pool's
        k, v = torch.cat([k, k[:3]]), torch.cat([v, v[:3]])
        slots = torch.cat([slots, torch.tensor([-1, c.kv.pool.shape[0] * 16, 1 << 40], device="cuda")])
    c.kv.write(slots, k, v)
    c.k[slots[:n]], c.v[slots[:n]] = k[:n], v[:n]
    after = c.kv.read(c.ints([0]), c.ints([0, 64]), 64)
    for got, want in zip(after, c.want(0)):
        same(got, want)
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[at] = False
    for a, b in zip(before, after):  # the tokens beside them keep theirs
        assert torch.equal(a[rest], b[rest])
    c.kv.check()


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page", [(128, 16), (80, 64), (8, 128), (24, 16)])
def test_ranges_of_sequences(dim, page, dtype, bits):
    lens = [300, 1, 0, 77, 16, 200]
    c = Pool(lens, dim=dim, page=page, dtype=dtype)
    kv = c.kv
    if bits == 16:
        from paper_2508_14544_gb300 import KVCache
        kv = KVCache(c.kv.pool.shape[0], page, 2, dim, len(lens) + 1, c.table.shape[1], dtype=c.dt)
        kv.pool.fill_(math.nan)
        for i, x in enumerate(lens):
            at = c.torch.from_numpy(c.slots(i, 0, x)).cuda()
            kv.write(at, c.k[at], c.v[at])
        for a, b in ((kv.table, c.kv.table), (kv.length, c.kv.length), (kv.ref, c.kv.ref)):
            a.copy_(b)
    entries = [(0, 0, 300), (0, 17, 40), (5, 15, 0), (2, 0, 0), (3, 76, 1), (0, 299, 1), (5, 31, 100), (1, 0, 1), (4, 3, 13)]  # sequence, first, tokens
    before, after = 3, 2  # rows of no entry
    cu = np.cumsum([before, *(n for _, _, n in entries)])
    n = int(cu[-1]) + after
    k, v = kv.read(c.ints([s for s, _, _ in entries]), c.ints(cu), n, first=c.ints([f for _, f, _ in entries]))
    for (s, f, x), a in zip(entries, cu):
        if bits == 4:
            wk, wv = c.want(s, f, f + x)
        else:
            at = c.torch.from_numpy(c.slots(s, f, f + x)).cuda()
            wk, wv = f64(c.k[at]), f64(c.v[at])
        same(k[a: a + x], wk)
        same(v[a: a + x], wv)
    for x in (k, v):
        assert not x[:before].any() and not x[n - after:].any()
    kv.check()


@pytest.mark.parametrize("bits", [4, 16])
def test_reads_that_are_refused_are_zeros(bits):
    from paper_2508_14544_gb300 import SimError
    c = Pool([40, 50], dim=64)
    kv = c.kv
    if bits == 16:
        from paper_2508_14544_gb300 import KVCache
        kv = KVCache(c.kv.pool.shape[0], 16, 2, 64, 3, c.table.shape[1])
        kv.pool.normal_()
        kv.table.copy_(c.kv.table)
        kv.length.copy_(c.kv.length)
    for seq, first, n in ((7, 0, 20), (-1, 0, 20), (0, 30, 11), (0, -1, 20), (2, 0, 1), (0, 2 ** 31 - 5, 10)):
        cu = c.ints([0, 10, 10 + n, 20 + n])
        k, v = kv.read(c.ints([0, seq, 1]), cu, 20 + n, first=c.ints([0, first, 3]))
        assert not k[10: 10 + n].any() and not v[10: 10 + n].any()
        a, _ = kv.read(c.ints([0, 1]), c.ints([0, 10, 20]), 20, first=c.ints([0, 3]))
        assert c.torch.equal(a[:10], k[:10]) and c.torch.equal(a[10:], k[10 + n:]) and a.any()
        with pytest.raises(SimError):
            kv.check()
    for cu in ([0, 30, 20], [-1, 10, 20], [0, 10, 21]):
        k, v = kv.read(c.ints([0, 1]), c.ints(cu), 20)
        assert not k.any() and not v.any()
        with pytest.raises(SimError):
            kv.check()
    kv.table[0, 1] = kv.pool.shape[0]  # a page that the pool does not have
    k, v = kv.read(c.ints([0]), c.ints([0, 40]), 40)
    assert not k[16:32].any() and not v[16:32].any() and k[:16].any() and k[32:].any()


def test_reading_many_entries():
    lens = [int(x) for x in np.random.default_rng(1).integers(0, 40, 1500)]
    c = Pool(lens, kv_heads=1, dim=32)
    cu = np.cumsum([0, *lens])
    k, v = c.kv.read(c.ints(range(1500)), c.ints(cu), int(cu[-1]))
    at = c.torch.from_numpy(np.concatenate([c.slots(i, 0, x) for i, x in enumerate(lens)])).cuda()
    same(k, held(f64(c.k[at]), "bfloat16"))
    same(v, held(f64(c.v[at]), "bfloat16"))


# ---- attention ------------------------------------------------------------------------------------------------------


def attend(c, queries, group, seqs=None, grouped=True, scale=None, spread=1.0, q=None, **more):
    n_q = int(sum(queries))
    if q is None:
        q = (c.torch.randn(n_q, c.heads * group, c.dim, generator=c.gen, device="cuda") * spread).to(c.dt)
    cu = c.ints([0, *np.cumsum(queries)])
    plan = c.kv.plan(c.ints(range(len(queries))) if seqs is None else seqs, cu, n_q, heads=c.heads * group, cu_group=c.bounds if grouped else None)
    return q, *c.kv.attend(q, plan, layer=c.layer, scale=scale, **more)


def check(c, queries, q, out, lse, scale=None):
    """The products of 16-bit floats are exact and summed in 32 bits, so the bounds are those of the 16-bit cache on the values held."""
    scale = c.dim ** -0.5 if scale is None else scale
    u, at = ROUND[c.dtype], 0
    q, out, lse = f64(q), f64(out), f64(lse)
    for i, t in enumerate(queries):
        n = c.lens[i]
        k, v = (x.transpose(1, 0, 2) for x in c.want(i))
        want, wl, mag = attention(q[at: at + t], k, v, scale)
        # P is rounded to 16 bits (and, in float16, below 2^-24 to multiples of that), the result again; sums and exponentials in 32 bits
        floor = n * 2.0 ** -25 * (np.abs(v).max() if n else 0) if c.dtype == "float16" else 0
        tol = 1.05 * u * (mag + np.abs(want)) + 2.0 ** -12 * mag + floor
        got = out[at: at + t]
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (i, n, t, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])
        none = np.isneginf(wl)
        assert np.array_equal(np.isneginf(lse[at: at + t]), none)
        assert np.all(np.abs(lse[at: at + t][~none] - wl[~none]) <= 2e-5 * np.maximum(1, np.abs(wl[~none]))), (i, n, t)
        at += t
    c.kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (80, 64), (8, 128), (72, 16), (96, 16), (128, 128)])
def test_single_tokens_over_many_lengths(dim, page, dtype):
    lens = [1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 130, 200, 255, 256, 257, 300, 511, 700]
    c = Pool(lens, dim=dim, page=page, dtype=dtype, seed=dim + page, layers=2)
    check(c, [1] * len(lens), *attend(c, [1] * len(lens), 4))


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (1, 7), (2, 8), (1, 9), (2, 16), (1, 17), (3, 33), (1, 64), (2, 65), (1, 129), (1, 300), (5, 3)])
def test_head_layouts(kv_heads, group):
    lens = [1, 40, 129, 300]
    c = Pool(lens, kv_heads=kv_heads, seed=group)
    check(c, [1] * 4, *attend(c, [1] * 4, group))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,queries,group", [
    ([5, 1, 130, 300], [5, 1, 130, 300], 1),        # whole prompts
    ([77, 300, 128], [20, 33, 128], 4),             # 80, 132, 512 rows
    ([500, 400], [37, 16], 8),                      # light remainders after heavy items
    ([64, 65, 200], [3, 0, 5], 5),                  # an entry without queries
    ([40, 50, 0, 60], [3, 2, 0, 5], 3),             # a few drafted tokens
    ([10, 3, 200], [12, 3, 9], 2),                  # rows that see nothing
])
def test_many_queries_see_the_keys_up_to_their_own(lens, queries, group, dim, dtype):
    c = Pool(lens, dim=dim, dtype=dtype, seed=len(lens))
    check(c, queries, *attend(c, queries, group))


def test_rows_behind_the_last_entry_and_empty_batches():
    c = Pool([30, 0, 20], dim=64)
    q = c.torch.randn(9, 8, 64, device="cuda").to(c.dt)
    plan = c.kv.plan(c.ints([0, 1, 2]), c.ints([2, 4, 5, 6]), 9, heads=8)
    out, lse = c.kv.attend(q, plan)
    for rows in (slice(0, 2), slice(4, 5), slice(6, 9)):  # of no entry, or of one without keys
        assert not out[rows].any() and c.torch.isneginf(lse[rows]).all()
    assert out[2:4].all() and out[5].all()
    plan = c.kv.plan(c.ints([]), c.ints([0]), 0, heads=8)
    out, _ = c.kv.attend(q[:0], plan)
    assert out.shape == (0, 8, 64)
    c.kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("grouped", [True, False])
@pytest.mark.parametrize("group", [4, 8])
def test_shared_prefixes(group, grouped, dtype):
    rng = np.random.default_rng(3)
    groups, prefix = [1, 30, 0, 25], 1024
    lens = [prefix + int(x) for x in rng.integers(1, 150, sum(groups))]
    queries = [int(x) for x in rng.integers(1, 4, len(lens))]
    c = Pool(lens, dim=128, page=32, dtype=dtype, groups=groups, prefix=prefix)
    check(c, queries, *attend(c, queries, group, grouped=grouped))


@pytest.mark.parametrize("group", [1, 8, 16])
@pytest.mark.parametrize("n", [20000, 131071])
def test_a_long_sequence_is_divided(n, group):
    c = Pool([n], kv_heads=1, dim=64, page=64, dtype="float16")
    check(c, [1], *attend(c, [1], group))
    check(c, [3], *attend(c, [3], group))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_flat_and_sharp_weights(spread, dtype):
    lens = [1, 100, 1000]
    c = Pool(lens, dim=128, dtype=dtype)
    queries = [1, 2, 1]
    check(c, queries, *attend(c, queries, 8, spread=spread))


def test_strides_alignment_scale_and_given_outputs():
    lens, queries = [100, 37], [1, 4]
    c = Pool(lens, dim=64)
    torch = c.torch
    x = torch.randn(5, 8, 64, device="cuda").to(c.dt)
    big = torch.zeros(5, 9, 65, dtype=c.dt, device="cuda")
    big[:, 1:, 1:] = x
    out = torch.full((5, 10, 72), 7.0, dtype=c.dt, device="cuda")
    q, o, lse = attend(c, queries, 4, q=big[:, 1:, 1:], scale=0.3, out=out[:, 1:9, :64])
    check(c, queries, x, o, lse, scale=0.3)
    assert (out[:, 0] == 7).all() and (out[:, 9] == 7).all() and (out[..., 64:] == 7).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("group,queries", [(4, 6), (2, 3), (40, 4)])
@pytest.mark.parametrize("which", ["keys", "values"])
def test_groups_that_are_not_finite_spoil_the_rows_that_see_them(which, group, queries, dtype):
    import torch
    n, dim = 150, 128
    c = Pool([n], kv_heads=1, dim=dim, dtype=dtype)
    at = n - 2  # seen by the last two queries
    slot = torch.from_numpy(c.slots(0, at, at + 1)).cuda()
    x = c.k if which == "keys" else c.v
    x[slot, 0, 37] = math.inf
    c.kv.write(slot, c.k[slot], c.v[slot])
    q, out, lse = attend(c, [queries], group)
    clean, wl, _ = attention(f64(q)[: queries - 2], *(y.transpose(1, 0, 2)[:, : n - 2] for y in c.want(0)), dim ** -0.5)
    assert np.abs(f64(out)[: queries - 2] - clean).max() < 0.1 and np.abs(f64(lse)[: queries - 2] - wl).max() < 1e-4
    spoilt = np.isnan(f64(out)[queries - 2:])
    if which == "keys":
        assert spoilt.all() and np.isnan(f64(lse)[queries - 2:]).all()
    else:
        assert spoilt[..., 32:64].all() and not spoilt[..., :32].any() and not spoilt[..., 64:].any()


@pytest.mark.parametrize("group,tokens", [(4, 1), (4, 5), (40, 1), (50, 6)])
@pytest.mark.parametrize("page", [16, 128])
def test_pages_that_the_pool_does_not_have_are_zeros(group, tokens, page):
    n = 5 * page - 3
    c = Pool([n], page=page, dim=80)
    for at, number in ((0, c.kv.pool.shape[0]), (2, 1 << 20), (3, -5)):
        c.kv.table[0, at] = number
        real = c.torch.from_numpy(c.slots(0, at * page, (at + 1) * page)).cuda()
        c.k[real], c.v[real] = 0, 0
    check(c, [tokens], *attend(c, [tokens], group))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_the_life_of_sequences(dtype):
    """Extended, forked inside a page, extended again (the shared page is copied), freed, compacted: then read and attended to."""
    import torch

    from paper_2508_14544_gb300 import KVCache
    dt, D, H = getattr(torch, dtype), 96, 2
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv = KVCache(64, 16, H, D, 8, 16, n_layers=2, dtype=dt, bits=4)
    kv.pool.fill_(0x7f)
    g = torch.Generator("cuda").manual_seed(3)
    have = {}

    def add(seqs, counts):
        cu = np.cumsum([0, *counts])
        slots = kv.extend(ints(seqs), ints(cu), int(cu[-1]))
        for layer in range(2):
            k, v = (torch.randn(int(cu[-1]), H, D, generator=g, device="cuda").to(dt) for _ in range(2))
            kv.write(slots, k, v, layer=layer)
            for s, a, b in zip(seqs, cu, cu[1:]):
                x = torch.stack([k[a:b], v[a:b]])
                have[s, layer] = torch.cat([have[s, layer], x], 1) if (s, layer) in have else x

    add([0, 1, 2], [37, 20, 5])
    kv.fork(ints([0, 0]), ints([3, 4]), tokens=ints([37, 21]))
    kv.copy(ints([1]), ints([5]))
    for d, s, n in ((3, 0, 37), (4, 0, 21), (5, 1, 20)):
        for layer in range(2):
            have[d, layer] = have[s, layer][:, :n]
    add([3, 4, 0, 5], [1, 30, 2, 1])
    kv.free(ints([1]))
    kv.free(ints([2]), ints([3]))
    have = {(s, layer): x[:, :3] if s == 2 else x for (s, layer), x in have.items() if s != 1}
    kv.compact()
    add([2], [4])
    kv.check()
    seqs = [0, 2, 3, 4, 5]
    lens = [have[s, 0].shape[1] for s in seqs]
    assert kv.length.tolist() == [39, 0, 7, 38, 51, 21, 0, 0]
    cu = np.cumsum([0, *lens])
    q = torch.randn(len(seqs), 8, D, generator=g, device="cuda").to(dt)
    plan = kv.plan(ints(seqs), ints(range(len(seqs) + 1)), len(seqs), heads=8)
    for layer in range(2):
        k, v = kv.read(ints(seqs), ints(cu), int(cu[-1]), layer=layer)
        out, lse = kv.attend(q, plan, layer=layer)
        for i, s in enumerate(seqs):
            wk, wv = (held(f64(x), dtype) for x in have[s, layer])
            same(k[cu[i]: cu[i + 1]], wk)
            same(v[cu[i]: cu[i + 1]], wv)
            want, wl, mag = attention(f64(q[i: i + 1]), wk.transpose(1, 0, 2), wv.transpose(1, 0, 2), D ** -0.5)
            assert (np.abs(f64(out[i]) - want[0]) <= 2.1 * ROUND[dtype] * mag[0] + 2.0 ** -12 * mag[0] + 2.0 ** -20).all()
            assert (np.abs(f64(lse[i]) - wl[0]) <= 1e-4).all()
    kv.check()


def test_a_captured_step_is_replayed():
    import torch
    c = Pool([50, 33], dim=128)
    kv, ints = c.kv, c.ints
    slots = torch.from_numpy(np.concatenate([c.slots(0, 49, 50), c.slots(1, 32, 33)])).cuda()
    k, v = (torch.randn(2, 2, 128, device="cuda").to(c.dt) for _ in range(2))
    q = torch.randn(2, 8, 128, device="cuda").to(c.dt)
    seqs, cu, cur = ints([0, 1]), ints([0, 1, 2]), ints([0, 50, 83])

    def step():
        kv.write(slots, k, v)
        plan = kv.plan(seqs, cu, 2, heads=8)
        return (*kv.attend(q, plan), *kv.read(seqs, cur, 83))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for turn in range(3):
        k.normal_()
        v.normal_()
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.k[slots], c.v[slots] = k, v
        check(c, [1, 1], q, got[0], got[1])
        same(got[2][:50], c.want(0)[0])
        same(got[3][50:], c.want(1)[1])


def test_calls_on_a_stream():
    import torch
    c = Pool([70], dim=64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k, v = c.kv.read(c.ints([0]), c.ints([0, 70]), 70, stream=side.cuda_stream)
    side.synchronize()
    same(k, c.want(0)[0])
    same(v, c.want(0)[1])


def test_results_do_not_change_from_run_to_run():
    lens = [1000, 3000, 77]
    c = Pool(lens, dim=128)
    q, out, lse = attend(c, [1, 1, 1], 8)
    for _ in range(3):
        _, o, s = attend(c, [1, 1, 1], 8, q=q)
        assert c.torch.equal(o, out) and c.torch.equal(s, lse)


def test_what_is_refused():
    import torch

    from paper_2508_14544_gb300 import KVCache, SimError
    c = Pool([70], dim=64)
    kv = c.kv
    with pytest.raises(ValueError):
        KVCache(8, 16, 2, 64, 4, 4, bits=8)
    with pytest.raises(ValueError):
        KVCache(8, 16, 2, 60, 4, 4, bits=4)
    args = kv.pool, kv.table, kv.length, kv.ref
    for more in ({}, dict(head_dim=64), dict(dtype=torch.float16), dict(head_dim=80, dtype=torch.float16), dict(head_dim=64, dtype=torch.float32)):
        with pytest.raises(ValueError):
            KVCache.wrap(*args, **more)
    again = KVCache.wrap(*args, head_dim=64, dtype=torch.bfloat16)
    same(again.read(c.ints([0]), c.ints([0, 70]), 70)[0], c.want(0)[0])
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    for bad in (x.half(), x.float(), x[:, :1], x[..., :32], x.clone().requires_grad_()):
        with pytest.raises(ValueError):
            kv.write(slots, bad, x)
    for bad in (c.ints([0]).long(), torch.zeros(1, dtype=torch.int32), c.ints([0, 0])):
        with pytest.raises(ValueError):
            kv.read(bad, c.ints([0, 70]), 70)
    with pytest.raises(SimError):
        kv.read(c.ints([0]), c.ints([0, 70]), 70, layer=1)
    with pytest.raises(SimError):
        kv.write(slots, x, x, layer=5)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page,heads,most", [(128, 16, 8, 200), (128, 64, 8, 700), (80, 32, 3, 500), (32, 16, 1, 900), (64, 128, 4, 300)])
def test_lists_of_many_tokens_in_any_order(dim, page, heads, most, dtype):
    """Sequences' tokens one after the other, so that strips begin anywhere in the list; some tokens without a slot, some out of order."""
    import torch

    from paper_2508_14544_gb300 import KVCache
    rng = np.random.default_rng(dim + page)
    lens = [int(x) for x in rng.integers(0, most, 60)]
    n_pages = sum(-(-x // page) for x in lens) + 5
    order = rng.permutation(n_pages)
    kv = KVCache(n_pages, page, heads, dim, 60, max(-(-x // page) for x in lens) + 1, n_layers=2, dtype=getattr(torch, dtype), bits=4)
    kv.pool.fill_(0xff)
    at, table, slots = 0, np.full(tuple(kv.table.shape), -1, np.int32), []
    for i, x in enumerate(lens):
        k = -(-x // page)
        table[i, :k] = order[at: at + k]
        at += k
        pos = np.arange(x)
        slots.append(table[i, pos // page].astype(np.int64) * page + pos % page)
    kv.table.copy_(torch.from_numpy(table))
    kv.length.copy_(torch.tensor(lens, dtype=torch.int32))
    flat = np.concatenate(slots)
    n = len(flat)
    where = np.arange(n)
    for a in rng.integers(0, n - 40, 8):  # pieces turned round
        where[a: a + 33] = where[a: a + 33][::-1].copy()
    none = rng.choice(n, 20, replace=False)
    listed = flat[where]
    k, v = (torch.randn(n, heads, dim, device="cuda", generator=torch.Generator("cuda").manual_seed(s)).to(kv.dtype) for s in (1, 2))
    gaps = listed.copy()
    gaps[none] = rng.choice([-1, -7, n_pages * page, 1 << 45], 20)
    kv.write(torch.from_numpy(gaps).cuda(), k, v, layer=1)
    at_none = torch.from_numpy(none).cuda()
    kv.write(torch.from_numpy(listed[none]).cuda(), k[at_none], v[at_none], layer=1)
    cu = np.cumsum([0, *lens])
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    rk, rv = kv.read(ints(range(60)), ints(cu), n, layer=1)
    back = np.empty(n, np.int64)
    back[where] = np.arange(n)
    back = torch.from_numpy(back).cuda()
    same(rk, held(f64(k[back]), dtype))
    same(rv, held(f64(v[back]), dtype))
    assert (kv.pool[:, 0] == 0xff).all()  # the other layer
    kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,page", [(128, 32), (80, 16), (24, 64), (64, 16)])
def test_the_pool_is_laid_out_as_the_header_says(dim, page, dtype):
    from paper_2508_14544_gb300 import _lib
    n, G, heads = 45, -(-dim // 32), 2
    c = Pool([n], kv_heads=heads, dim=dim, page=page, dtype=dtype, fill=0)
    assert tuple(c.kv.pool.shape[1:]) == (1, 2, heads, page, 20 * G) and c.kv.bits == 4
    assert c.kv.pool.numel() == _lib.lib().sim_kv_pool_bytes(c.kv._ref)
    pool = c.kv.pool.cpu().numpy().reshape(-1, 2, heads, page // 16, 320 * G)
    got = np.zeros((2, n, heads, dim))

    def number(strip, at):  # a 16-bit float
        bits = np.array([int(strip[at]) | int(strip[at + 1]) << 8], np.uint32)
        return float((bits << 16).view(np.float32)[0]) if dtype == "bfloat16" else float(bits.astype(np.uint16).view(np.float16)[0])
    for t in range(n):
        where = pool[c.table[0, t // page], :, :, t % page // 16]
        T = t % 16
        for h in range(heads):
            k, v = where[0, h], where[1, h]
            for i in range(dim):
                g, d = divmod(i, 32)
                at = 16 * G * T + 4 * G * (d // 8) + 4 * g
                code = int.from_bytes(k[at: at + 4].tobytes(), "little") >> (4 * (d % 8 // 2) + 16 * (d % 2)) & 15
                at = 256 * G + 4 * G * T + 4 * g
                got[0, t, h, i] = number(k, at + 2) + code * number(k, at)
                at = 128 * G * (T // 8) + 4 * G * (4 * (d // 4) + T % 8 // 2) + 4 * g + 2 * (T % 2)
                code = int.from_bytes(v[at: at + 2].tobytes(), "little") >> (4 * (d % 4)) & 15
                at = 256 * G + 8 * G * (T // 2) + 8 * g + 2 * (T % 2)
                got[1, t, h, i] = number(v, at + 4) + code * number(v, at)
    for x, want in zip(got, c.want(0)):
        assert np.array_equal(round16(x, dtype), want)
