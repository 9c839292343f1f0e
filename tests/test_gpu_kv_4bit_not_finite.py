"""Groups of a 4-bit cache that are not numbers: they spoil their own columns of the rows that see them, and nothing else."""
import math

import numpy as np
import pytest

from tests.kv_reference import attention
from tests.test_gpu_kv_4bit import ROUND, Pool, attend, f64

pytestmark = pytest.mark.gpu


def right(c, t, q, out, lse, bad):
    """The last t tokens' rows of sequence 0: columns of groups in `bad` (token, group) that a row sees are not numbers, the others what the held
    values give.  Tolerances: P is rounded to the cache's type (in float16 below 2^-24 to multiples of that), the result again; sums in 32 bits."""
    n, u = c.lens[0], ROUND[c.dtype]
    k, v = (x.transpose(1, 0, 2) for x in c.want(0))
    spoilt = np.zeros(out.shape, bool)
    for token, g in bad:
        assert np.isnan(v[:, token, 32 * g: 32 * g + 32]).all()
        spoilt[max(token - (n - t), 0):, :, 32 * g: 32 * g + 32] = True
    v = np.nan_to_num(v, nan=0.0)
    want, wl, mag = attention(f64(q), k, v, c.dim ** -0.5)
    floor = n * 2.0 ** -25 * np.abs(v).max() if c.dtype == "float16" else 0
    got = f64(out)
    assert np.array_equal(np.isnan(got), spoilt)
    wrong = ~(np.abs(got - want) <= 1.05 * u * (mag + np.abs(want)) + 2.0 ** -12 * mag + floor) & ~spoilt
    assert not wrong.any(), (np.argwhere(wrong)[:4].tolist(), got[wrong][:4], want[wrong][:4])
    assert (np.abs(f64(lse) - wl) <= 2e-5 * np.maximum(1, np.abs(wl))).all()
    c.kv.check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
@pytest.mark.parametrize("group,tokens", [(2, 3), (4, 6), (9, 4), (40, 4), (66, 4), (100, 3), (3, 100)])  # light, and heavy with and without light rows
@pytest.mark.parametrize("n", [120, 150, 400])
def test_the_other_groups_of_a_token_keep_their_values(n, group, tokens, dim, dtype):
    """Tokens that only some of an item's rows see, one of them with nearly all of their weight, have groups that are not numbers."""
    import torch
    c = Pool([n], kv_heads=1, dim=dim, dtype=dtype, seed=n + dim)
    last = -(-dim // 32) - 1
    bad = [(n - 2, 1), (n - 1, 0), (n - tokens, last)]
    towards = torch.randn(dim, generator=c.gen, device="cuda")
    at = torch.from_numpy(c.slots(0, 0, n)).cuda()
    c.k[at[n - 2], 0] = (2 * towards).to(c.dt)
    for token, g in bad:
        c.v[at[token], 0, 32 * g + 5] = math.inf if g else math.nan
    c.kv.write(at, c.k[at], c.v[at])
    q = (towards + 0.1 * torch.randn(tokens, group, dim, generator=c.gen, device="cuda")).to(c.dt)
    _, out, lse = attend(c, [tokens], group, q=q)
    right(c, tokens, q, out, lse, bad)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("group,tokens", [(4, 3), (50, 3)])
def test_a_group_that_all_rows_see(group, tokens, dtype):
    import torch
    n = 300
    c = Pool([n], kv_heads=1, dim=96, dtype=dtype)
    bad = [(7, 2), (200, 0)]
    for token, g in bad:
        slot = torch.from_numpy(c.slots(0, token, token + 1)).cuda()
        c.v[slot, 0, 32 * g] = math.nan
        c.kv.write(slot, c.k[slot], c.v[slot])
    q, out, lse = attend(c, [tokens], group)
    right(c, tokens, q, out, lse, bad)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("group,tokens", [(1, 1), (8, 1), (8, 3), (40, 2)])
@pytest.mark.parametrize("what", ["query", "last value", "first value", "last key"])
def test_rows_in_many_pieces(what, group, tokens, dtype):
    """Some 157 tiles of keys on all SMs: what is not a number in one piece of a row comes through the joining of all of them."""
    import torch
    n, dim = 20000, 64
    c = Pool([n], kv_heads=1, dim=dim, page=64, dtype=dtype)
    q, out, lse = attend(c, [tokens], group)
    clean_o, clean_l = out.clone(), lse.clone()
    if what == "query":
        q[tokens - 1, 0, 3] = math.nan
    else:
        at = torch.from_numpy(c.slots(0, 0, 1) if what == "first value" else c.slots(0, n - 1, n)).cuda()
        x = c.k if what == "last key" else c.v
        x[at, 0, 40] = math.nan
        c.kv.write(at, c.k[at], c.v[at])
    _, out, lse = attend(c, [tokens], group, q=q)
    odd_o, odd_l = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
    if what == "query":
        odd_o[-1, 0], odd_l[-1, 0] = True, True
    elif what == "last key":
        odd_o[-1], odd_l[-1] = True, True
    else:
        odd_o[-1 if what == "last value" else 0:, :, 32:] = True
    assert torch.equal(out.isnan(), odd_o) and torch.equal(lse.isnan(), odd_l)
    if what == "query":  # the other rows: the same bits
        assert torch.equal(out[~odd_o], clean_o[~odd_o]) and torch.equal(lse[~odd_l], clean_l[~odd_l])
    elif what == "last key":
        assert torch.equal(out[:-1], clean_o[:-1]) and torch.equal(lse[:-1], clean_l[:-1])
    else:
        right(c, tokens, q, out, lse, [(n - 1 if what == "last value" else 0, 1)])
    c.kv.check()
