"""Values that are infinite or not a number, in long sequences: they reach the queries that see them and no others, and no
block gives up its work over them."""
import math

import pytest

pytestmark = pytest.mark.gpu
H, G, D, P, N, T = 8, 8, 128, 128, 131072, 1024  # one sequence of N tokens, the last T of them queries: 256 rows an item


@pytest.fixture(scope="module")
def long_chunk():
    import torch

    from paper_2508_14544_gb300 import KVCache
    g = torch.Generator("cuda").manual_seed(11)
    pool = torch.empty(N // P, 1, 2, H, P, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv = KVCache.wrap(pool, torch.arange(N // P, dtype=torch.int32, device="cuda")[None], ints([N]), torch.ones(N // P, dtype=torch.int32, device="cuda"))
    q = torch.empty(T, H * G, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return kv, q, kv.plan(ints([0]), ints([0, T]), T, heads=H * G)


def right(kv, q, out, token, head, columns):
    """One row against 64 bits, in the columns given."""
    x = kv.pool[:, 0, :, head // G].double().permute(1, 0, 2, 3).reshape(2, N, D)[:, : N - T + token + 1]
    s = x[0] @ q[token, head].double() / math.sqrt(D)
    w = s.softmax(0)
    v = x[1][:, columns]
    want, mag = w @ v, w @ v.abs()
    # P is rounded to bfloat16 and the result again; sums in 32 bits
    assert ((out[token, head, columns].double() - want).abs() <= 1.05 * 2.0 ** -8 * (mag + want.abs()) + 2.0 ** -12 * mag).all()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_values_that_rows_of_the_same_item_do_not_see(long_chunk, bad):
    """The last of each 32 tokens (an item's) has such a value, in a column of its own."""
    import torch
    kv, q, plan = long_chunk
    values = kv.pool[:, 0, 1].permute(0, 2, 1, 3).reshape(N, H, D)  # a copy: written back below
    tokens = torch.arange(31, T, 32, device="cuda")
    at = N - T + tokens
    was = values[at, :, tokens // 32].clone()
    kv.pool[at // P, 0, 1, :, at % P, tokens // 32] = bad
    out, lse = kv.attend(q, plan)
    kv.check()
    token, column = torch.arange(T, device="cuda")[:, None, None], torch.arange(D, device="cuda")[None, None]
    assert torch.equal(~torch.isfinite(out), (column * 32 + 31 <= token).expand(T, H * G, D)) and torch.isfinite(lse).all()
    for t, h in ((0, 0), (30, 63), (31, 8), (32, 9), (500, 17), (1022, 40), (1023, 63)):
        right(kv, q, out, t, h, [c for c in range(D) if c * 32 + 31 > t])
    kv.pool[at // P, 0, 1, :, at % P, tokens // 32] = was


@pytest.mark.parametrize("what", ["value", "query", "key"])
def test_what_rows_see_themselves(long_chunk, what):
    import torch
    kv, q, plan = long_chunk
    q = q.clone()
    was = kv.pool[0, 0].clone()
    finite = torch.ones(T, H * G, D, dtype=torch.bool, device="cuda")
    if what == "value":  # of head 3, in one column each
        kv.pool[0, 0, 1, 3, 5, 7], kv.pool[0, 0, 1, 3, 6, 70] = math.nan, math.inf
        finite[:, 3 * G: 4 * G, [7, 70]] = False
    elif what == "key":
        kv.pool[0, 0, 0, 3, 5, 7] = math.nan
        finite[:, 3 * G: 4 * G] = False
    else:
        q[100, 5, 1] = math.nan
        finite[100, 5] = False
    out, lse = kv.attend(q, plan)
    kv.check()
    assert torch.equal(torch.isfinite(out), finite)
    for t, h in ((0, 0), (77, 25), (100, 6), (1023, 63)):
        right(kv, q, out, t, h, finite[t, h].nonzero()[:, 0].tolist())
    kv.pool[0, 0] = was
