"""Attention over stretches of keys so long that sums of 32 bits and waits have to be looked after: every block has a whole
sequence of its own (all of them on the same pages) or more."""
import math

import pytest

pytestmark = pytest.mark.gpu
ROUND = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}  # unit roundoff: 8 and 11 bits


def cache(pool, n, sequences):
    import torch

    from paper_2508_14544_gb300 import KVCache
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(pool.shape[0], dtype=torch.int32, device="cuda")[None].expand(sequences, -1).contiguous()
    return KVCache.wrap(pool, table, ints([n] * sequences), ints([sequences] * pool.shape[0])), ints


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,group", [(1, 8), (2, 128)])  # rows of light and of heavy items
@pytest.mark.parametrize("n", [2 ** 17 + 5, 2 ** 20 + 77])
def test_values_of_one_sign_with_equal_weights(n, tokens, group, dtype):
    import torch
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    sequences = 2 * sms if tokens == 1 else sms
    g = torch.Generator("cuda").manual_seed(3)
    pool = torch.zeros(-(-n // 128), 1, 2, 1, 128, 8, dtype=getattr(torch, dtype), device="cuda")
    pool[:, :, 1] = 0.5 + torch.rand(pool[:, :, 1].shape, generator=g, device="cuda").to(pool.dtype)
    kv, ints = cache(pool, n, sequences)
    q = torch.randn(sequences * tokens, group, 8, generator=g, device="cuda").to(pool.dtype)
    plan = kv.plan(ints(range(sequences)), ints(range(0, sequences * tokens + 1, tokens)), sequences * tokens, heads=group)
    out, lse = kv.attend(q, plan)
    kv.check()
    v = pool[:, 0, 1, 0].reshape(-1, 8).double()
    for t in range(tokens):
        see = n - tokens + 1 + t
        want = v[:see].mean(0)
        # the result is rounded, the sums in 32 bits lose no more than another 2^-12
        assert ((out[t::tokens].double() - want).abs() <= (ROUND[dtype] + 2.0 ** -12) * want).all()
        assert ((lse[t::tokens].double() - math.log(see)).abs() <= 2e-5 * math.log(see)).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("tokens,group", [(1, 8), (20, 1), (1, 64), (40, 6)])
@pytest.mark.parametrize("n", [32768, 32768 + 11, 3 * 32768 + 300])
def test_scores_that_change_along_the_keys(n, tokens, group, bad, dtype):
    """Ranges of keys with weights far apart, the last ones seen by some of the rows; there also values that are not finite."""
    import torch
    sms, D = torch.cuda.get_device_properties(0).multi_processor_count, 72
    sequences = 2 * sms if tokens * group <= 32 else sms
    g = torch.Generator("cuda").manual_seed(4)
    pool = torch.randn(-(-n // 64), 1, 2, 1, 64, D, generator=g, device="cuda")
    pool[:, :, 0] *= torch.linspace(0.2, 2.0, pool.shape[0], device="cuda").roll(200)[:, None, None, None, None]
    pool = pool.to(getattr(torch, dtype))
    if bad and tokens > 1:
        for x in (n - tokens // 2, n - 2):
            pool[x // 64, 0, 1, 0, x % 64, x % D] = math.inf
    kv, ints = cache(pool, n, sequences)
    q = torch.randn(sequences * tokens, group, D, generator=g, device="cuda").to(pool.dtype)
    out, lse = kv.attend(q, kv.plan(ints(range(sequences)), ints(range(0, sequences * tokens + 1, tokens)), sequences * tokens, heads=group))
    kv.check()
    k, v = pool[:, 0, :, 0].transpose(0, 1).reshape(2, -1, D)[:, :n].double()
    u = ROUND[dtype]
    for i in (0, 1, sequences - 1):
        x = q[i * tokens: (i + 1) * tokens].double()
        s = torch.einsum("tgd,sd->tgs", x, k) / math.sqrt(D)
        see = torch.arange(n, device="cuda") <= torch.arange(n - tokens, n, device="cuda")[:, None]
        s = s.masked_fill(~see[:, None], -math.inf)
        w, fine = s.softmax(-1), torch.isfinite(v)
        infinite = torch.einsum("ts,sd->td", see.double(), (~fine).double()) > 0
        y = torch.where(fine, v, 0.0)
        want, mag = torch.einsum("tgs,sd->tgd", w, y), torch.einsum("tgs,sd->tgd", w, y.abs())
        got, at = out[i * tokens: (i + 1) * tokens].double(), infinite[:, None].expand_as(want)
        floor = n * 2.0 ** -25 * y.abs().max() if dtype == "float16" else 0
        assert not torch.isfinite(got[at]).any() and torch.isfinite(got[~at]).all()
        assert (((got - want).abs() <= 1.05 * u * (mag + want.abs()) + 2.0 ** -12 * mag + floor) | at).all()
        wl = s.logsumexp(-1)
        assert ((lse[i * tokens: (i + 1) * tokens].double() - wl).abs() <= 2e-5 * wl.abs().clamp(min=1)).all()


def test_a_stretch_that_takes_longer_than_a_wait_may():
    """190 million keys of one head for 304 tokens with 128 query heads, an item of two tokens for each of 152 SMs: no wait
    of a block, a second or so each, is for the whole of it.  Values of one: every sum is exact up to 2^24, the joint result
    is one up to its rounding."""
    import torch
    n, t = 190_000_000 // 128 * 128 + 77, 304
    pool = torch.zeros(-(-n // 128), 1, 2, 1, 128, 8, dtype=torch.bfloat16, device="cuda")  # 6 GB
    pool[:, :, 1] = 1
    kv, ints = cache(pool, n, 1)
    q = torch.randn(t, 128, 8, device="cuda").bfloat16()
    plan = kv.plan(ints([0]), ints([0, t]), t, heads=128)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, lse = kv.attend(q, plan)
    end.record()
    kv.check()
    assert (out == 1).all()
    want = torch.log(torch.arange(n - t + 1, n + 1, dtype=torch.float64, device="cuda"))[:, None]
    assert ((lse - want).abs() <= 2e-5 * want).all()
    assert begin.elapsed_time(end) > 1450  # ms: 2e9 cycles, the longest wait, at 1380 MHz or more; else this shows nothing
