"""The cache's pages on the GPU against Python lists: metadata, slots and contents, whole."""
import numpy as np
import pytest

from tests.kv_reference import Pages

pytestmark = pytest.mark.gpu


class Both:
    """A KVCache and its reference, driven by the same calls."""

    def __init__(self, n_pages, page, max_seqs, max_pages, heads=2, dim=16, layers=2, dtype="bfloat16"):
        import torch

        from paper_2508_14544_gb300 import KVCache
        self.torch = torch
        self.kv = KVCache(n_pages, page, heads, dim, max_seqs, max_pages, n_layers=layers, dtype=getattr(torch, dtype))
        self.kv.pool.zero_()
        self.ref = Pages(n_pages, page, max_seqs, max_pages)
        self.heads, self.dim, self.layers, self.seen = heads, dim, layers, 0

    def ints(self, x):
        return self.torch.tensor(list(x), dtype=self.torch.int32, device="cuda")

    def extend(self, seqs, new, n_new=None):
        cu = [0, *np.cumsum(new).tolist()]
        return self.extend_cu(seqs, cu, cu[-1] if n_new is None else n_new)

    def extend_cu(self, seqs, cu, n_new):
        got = self.kv.extend(self.ints(seqs), self.ints(cu), n_new)
        want = self.ref.extend(list(seqs), cu, n_new)
        assert got.tolist() == want
        # each token's keys are a number of its own below 256 (exact in 16 bits), by head, layer and column
        self.seen += 1
        values = [(self.seen * 37 + x * 11) % 251 for x in range(n_new)]
        t = self.torch
        x = t.tensor(values, dtype=t.float32, device="cuda")[:, None, None]
        h = t.arange(self.heads, device="cuda")[None, :, None]
        c = t.arange(self.dim, device="cuda")[None, None]
        for layer in range(self.layers):
            k = ((x + 3 * h + 5 * c + 7 * layer) % 251).to(self.kv.dtype)
            self.kv.write(got, k, -k, layer=layer)
        self.ref.write(want, values)

    def call(self, name, *lists):
        args = [None if x is None else self.ints(x) for x in lists]
        getattr(self.kv, name)(*args)
        getattr(self.ref, name)(*[None if x is None else list(x) for x in lists])

    def compact(self):
        assert self.kv.compact().tolist() == self.ref.compact()

    def same(self, code=0):
        from paper_2508_14544_gb300 import SimError
        r, kv = self.ref, self.kv
        assert np.array_equal(kv.table.cpu().numpy(), r.table())
        assert kv.length.tolist() == r.length
        assert kv.ref.tolist() == r.ref
        pool = kv.pool.float().cpu().numpy()  # [page, layer, 2, head, token, column]
        for s, row in enumerate(r.rows):
            for j, p in enumerate(row):
                n = min(r.P, r.length[s] - j * r.P)
                x = r.data[p, :n]
                for layer in range(self.layers):
                    want = (x[None, :, None] + 3 * np.arange(self.heads)[:, None, None] + 5 * np.arange(self.dim) + 7 * layer) % 251
                    assert np.array_equal(pool[p, layer, 0, :, :n], want), (s, j, layer)
                    assert np.array_equal(pool[p, layer, 1, :, :n], -want), (s, j, layer)
        assert r.refused == code
        if code:
            with pytest.raises(SimError) as e:
                kv.check()
            assert e.value.code == code
            r.refused = 0
        kv.check()


@pytest.mark.parametrize("page,dtype,heads,dim,layers", [(16, "bfloat16", 2, 16, 2), (32, "float16", 3, 40, 1), (64, "bfloat16", 1, 8, 3),
                                                         (128, "float16", 1, 128, 1)])
def test_a_random_life(page, dtype, heads, dim, layers):
    rng = np.random.default_rng(page)
    b = Both(97, page, 23, 7, heads, dim, layers, dtype)
    for step in range(60):
        kind = rng.integers(0, 6)
        live = [s for s in range(23) if b.ref.length[s]]
        empty = [s for s in range(23) if not b.ref.length[s]]
        n = int(rng.integers(1, 8))
        if kind <= 1:
            seqs = rng.permutation(23)[:n].tolist()
            b.extend(seqs, rng.integers(0, 2 * page + 2, n).tolist() if kind else [1] * n)
        elif kind == 2 and live:
            seqs = rng.permutation(live)[:n].tolist()
            b.call("free", seqs, None if rng.random() < 0.5 else rng.integers(0, 3 * page, len(seqs)).tolist())
        elif kind == 3 and live and empty:
            dst = rng.permutation(empty)[:n].tolist()
            src = rng.choice(live, len(dst)).tolist()
            b.call("fork", src, dst, None if rng.random() < 0.5 else [int(rng.integers(0, b.ref.length[s] + 1)) for s in src])
        elif kind == 4 and live and empty:
            dst = rng.permutation(empty)[:2].tolist()
            b.call("copy", rng.choice(live, len(dst)).tolist(), dst)
        elif kind == 5:
            b.compact()
        b.same(b.ref.refused)


def test_many_sequences_and_pages():
    """More entries than a block has threads, and more pages than its warps take in one walk."""
    rng = np.random.default_rng(5)
    b = Both(9001, 16, 2500, 40, heads=1, dim=8, layers=1)
    b.extend(rng.permutation(2500).tolist(), rng.integers(0, 60, 2500).tolist())
    b.same()
    b.call("free", rng.permutation(2500)[:1300].tolist(), None)
    b.compact()
    b.same()
    empty = [s for s in range(2500) if not b.ref.length[s]]
    live = [s for s in range(2500) if b.ref.length[s]]
    b.call("fork", rng.choice(live, 1100).tolist(), empty[:1100], None)
    b.extend(empty[:1100], [1] * 1100)
    b.same()


def test_a_page_that_all_its_holders_extend():
    """Each of them copies it, and it becomes free."""
    b = Both(8, 16, 4, 4)
    b.extend([0], [20])
    b.call("fork", [0, 0], [1, 2], None)
    b.extend([2, 0, 1], [1, 1, 13])
    b.same()
    b.call("fork", [1], [3], [16])  # ends with a whole page: no copy
    b.extend([3, 1], [1, 1])
    b.same()


def test_no_pages_left_changes_nothing():
    b = Both(5, 16, 8, 4)
    b.extend([0, 1], [40, 16])
    b.extend([2, 3], [16, 1])
    b.same(-6)
    b.extend([2], [16])
    b.call("copy", [0], [3])
    b.same(-6)
    b.call("fork", [2] * 5, [3, 4, 5, 6, 7], [9] * 5)  # a shared page that five want to copy, and none is free
    b.extend([2, 3, 4, 5, 6, 7], [0, 1, 1, 1, 1, 1])
    b.same(-6)


def test_entries_that_are_refused():
    b = Both(40, 16, 6, 3)
    b.extend([0, 7, 1, -1, 2], [5, 5, 5, 5, 5])          # out of range
    b.same(-1)
    b.extend([0, 3, 0], [1, 2, 1])                        # repeated
    b.same(-1)
    b.extend([0, 4], [44, 48])                            # past max_pages
    b.same(-1)
    b.extend_cu([0, 1, 2], [0, 4, 2, 5], 5)               # offsets that decrease
    b.same(-1)
    b.extend_cu([0, 1], [0, 2, 9], 5)                     # and that pass the tokens there are
    b.same(-1)
    b.call("free", [0, 0, 1, 9], [1, 1, -3, 0])
    b.same(-1)
    b.call("fork", [1, 1, 2, 9, 1], [5, 1, 4, 3, 3], None)  # dst that is a src, not empty, src out of range, dst twice
    b.same(-1)
    b.call("free", [4, 5], None)
    b.call("fork", [1, 2], [5, 4], [99, 0])               # more tokens than there are
    b.same(-1)
    b.call("copy", [0, 1], [5, 2], )                      # not empty
    b.same(-1)


def test_entries_without_tokens_and_empty_calls():
    b = Both(10, 16, 4, 4)
    b.extend([], [])
    b.extend([1, 0], [0, 0])
    b.call("free", [], None)
    b.call("free", [2], [7])
    b.compact()
    b.same()
    b.extend([1, 0], [16, 0])
    b.extend_cu([0], [2, 4], 6)  # tokens before and after the only entry's: no slot
    b.same()


@pytest.mark.parametrize("token,head,offset", [(None, None, 0), (100, 40, 0), (97, 33, 1), (48, 16, 3)])
def test_write_from_strided_and_unaligned_tensors(token, head, offset):
    import torch

    from paper_2508_14544_gb300 import KVCache
    kv = KVCache(6, 16, 3, 16, 2, 6, dtype=torch.float16)
    kv.pool.zero_()
    n = 37
    raw = torch.randn(n * 128 + 64, device="cuda", dtype=torch.float16)
    k = torch.randn(n, 3, 16, device="cuda", dtype=torch.float16) if token is None else raw.as_strided((n, 3, 16), (token, head, 1), offset)
    v = raw.as_strided((n, 3, 16), (80, 20, 1), 5)
    slots = kv.extend(torch.tensor([1], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    slots[4] = -1
    slots[9] = 6 * 16
    kv.write(slots, k, v)
    x = kv.pool[:, 0].permute(1, 0, 3, 2, 4).reshape(2, -1, 3, 16)[:, :n]
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[[4, 9]] = False
    assert torch.equal(x[0][keep], k[keep]) and torch.equal(x[1][keep], v[keep])
    assert not x[:, ~keep].any()
    kv.check()


def test_offsets_past_32_bits():
    """Pages whose bytes and elements lie past 2^32: written, copied, moved."""
    import torch

    from paper_2508_14544_gb300 import KVCache
    kv = KVCache(2100, 128, 8, 128, 4, 4, n_layers=4)  # 2 MB a page, 2.2e9 elements
    first = 2090
    kv.ref[:first] = 1
    seqs, cu = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    slots = kv.extend(seqs, cu, 300)
    assert slots[0].item() == first * 128
    k = torch.randn(300, 8, 128, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(300, 8, 128, device="cuda", dtype=torch.bfloat16)
    for layer in (0, 3):
        kv.write(slots, k, v, layer=layer)
    kv.copy(seqs, seqs + 1)
    kv.ref[:first] = 0
    kv.compact()
    assert kv.table[:2, :3].tolist() == [[0, 1, 2], [3, 4, 5]]
    for row in kv.table[:2, :3].long():
        for layer in (0, 3):
            x = kv.pool[row, layer].permute(1, 0, 3, 2, 4).reshape(2, -1, 8, 128)[:, :300]
            assert torch.equal(x[0], k) and torch.equal(x[1], v)
    kv.check()


def test_in_a_graph_and_on_another_stream():
    import torch

    b = Both(50, 16, 6, 6)
    b.extend([0, 1, 2], [17, 16, 3])
    seqs, cu = b.ints([0, 1, 2]), b.ints([0, 1, 2, 3])
    k = torch.zeros(3, 2, 16, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        slots = b.kv.extend(seqs, cu, 3)
        for layer in range(2):
            b.kv.write(slots, k, k, layer=layer)
    torch.cuda.current_stream().wait_stream(side)
    want = b.ref.extend([0, 1, 2], [0, 1, 2, 3], 3)
    assert slots.tolist() == want
    with torch.cuda.stream(side):  # named by the caller instead
        torch.cuda.synchronize()
    slots = b.kv.extend(seqs, cu, 3, stream=side.cuda_stream)
    side.synchronize()
    assert slots.tolist() == b.ref.extend([0, 1, 2], [0, 1, 2, 3], 3)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        slots = b.kv.extend(seqs, cu, 3)
    for _ in range(15):
        graph.replay()
        assert slots.tolist() == b.ref.extend([0, 1, 2], [0, 1, 2, 3], 3)
    assert b.kv.length.tolist() == b.ref.length and np.array_equal(b.kv.table.cpu().numpy(), b.ref.table())
    b.kv.check()
