"""A table with page numbers that the pool does not have: these pages are zeros, and nothing else is read in their place."""
import numpy as np
import pytest

from tests.kv_reference import attention
from tests.test_gpu_kv_attend import ROUND, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("group,tokens", [(4, 1), (4, 5), (40, 1), (50, 6)])  # rows of light and of heavy items
def test_pages_that_the_pool_does_not_have_are_zeros(group, tokens, page, dim, dtype):
    n = 5 * page - 3
    c = Case([n], [tokens], group=group, dim=dim, page=page, dtype=dtype, seed=group)
    pages = c.kv.pool.shape[0]
    for at, number in ((0, pages), (2, 1 << 20), (3, -5)):
        c.kv.table[0, at] = number
    out, lse = c.run()
    rows = c.torch.from_numpy(c.table[0][:5].astype(np.int64)).cuda()
    kv = c.kv.pool[rows, 0].double()
    kv[[0, 2, 3]] = 0
    kv = kv.cpu().numpy().transpose(1, 2, 0, 3, 4).reshape(2, 2, -1, dim)[:, :, :n]
    want, wl, mag = attention(c.q.double().cpu().numpy(), kv[0], kv[1], dim ** -0.5)
    # P is rounded to 16 bits and the result again, sums in 32 bits; in float16 P has steps of 2^-24 at most
    tol = 1.05 * ROUND[dtype] * (mag + np.abs(want)) + 2.0 ** -12 * mag + (n * 2.0 ** -25 * np.abs(kv[1]).max() if dtype == "float16" else 0)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - wl) <= 2e-5 * np.maximum(1, np.abs(wl))).all()
    c.kv.check()
