"""Many small weights beside a large one: none of them is lost to the type that the probabilities are rounded to."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("group", [8, 64])  # rows of light and of heavy items
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("gap", [9.0, 14.0, 17.4])
def test_a_key_that_takes_nearly_all(gap, first, group, dtype):
    """One key with a value of zero, `gap` above 32767 others with values of one sign: the result is what these give."""
    import torch

    from paper_2508_14544_gb300 import KVCache
    n, D, sms = 32768, 64, torch.cuda.get_device_properties(0).multi_processor_count
    sequences = 2 * sms if group == 8 else sms  # one for each block
    g = torch.Generator("cuda").manual_seed(5)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = torch.zeros(n // 128, 1, 2, 1, 128, D, device="cuda")
    pool[:, 0, 0, 0, :, 0] = torch.rand(n // 128, 128, generator=g, device="cuda") - 0.5
    pool[:, 0, 1] = 0.5 + torch.rand(pool[:, 0, 1].shape, generator=g, device="cuda")
    page, token = (0, 3) if first else (200, 77)
    pool[page, 0, :, 0, token] = 0
    pool[page, 0, 0, 0, token, 0] = gap
    pool = pool.to(getattr(torch, dtype))
    q = torch.zeros(sequences, group, D, dtype=pool.dtype, device="cuda")
    q[:, :, 0] = 8
    kv = KVCache.wrap(pool, torch.arange(n // 128, dtype=torch.int32, device="cuda")[None].expand(sequences, -1).contiguous(), ints([n] * sequences),
                      ints([sequences] * (n // 128)))
    out, lse = kv.attend(q, kv.plan(ints(range(sequences)), ints(range(sequences + 1)), sequences, heads=group))
    kv.check()
    k, v = pool[:, 0, :, 0].transpose(0, 1).reshape(2, n, D).double()
    s = k[:, 0] * 8 / math.sqrt(D)
    want = s.softmax(0) @ v
    # P to its unit roundoff, in float16 to half a step of 2^-31 at least, and the result; sums in 32 bits
    u = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -11
    floor = 2.0 ** -32 * v.sum(0) if dtype == "float16" else 0
    assert ((out.double() - want).abs() <= 1.05 * u * 2 * want + 2.0 ** -12 * want + floor).all()
    assert ((lse.double() - s.logsumexp(0)).abs() <= 2e-5 * s.logsumexp(0)).all()
