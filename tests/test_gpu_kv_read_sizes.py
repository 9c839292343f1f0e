"""KVCache.read at the ends of its sizes."""
import numpy as np
import pytest

from tests.kv_4bit_reference import held
from tests.test_gpu_kv_4bit import Pool, f64, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [-1, 1 << 31, (1 << 32) + 20, 1 << 40])
def test_more_rows_than_a_call_has_are_refused(n):
    """(2^32 + 20 would otherwise be taken for 20, and the rows behind them left as they were.)"""
    c = Pool([20], kv_heads=1, dim=8)
    with pytest.raises(ValueError):
        c.kv.read(c.ints([0]), c.ints([0, 20]), n)
    c.kv.check()


@pytest.mark.parametrize("bits", [4, 16])
def test_as_many_entries_as_a_call_has(bits):
    """2^17 entries of zero to three tokens of the same few sequences."""
    import torch
    lens = [50, 7, 300]
    c = Pool(lens, kv_heads=1, dim=40)
    kv = c.kv
    if bits == 16:
        from paper_2508_14544_gb300 import KVCache
        kv = KVCache(c.kv.pool.shape[0], 16, 1, 40, 4, c.table.shape[1])
        kv.table.copy_(c.kv.table)
        kv.length.copy_(c.kv.length)
        at = torch.from_numpy(np.concatenate([c.slots(i, 0, x) for i, x in enumerate(lens)])).cuda()
        kv.write(at, c.k[at], c.v[at])
    rng = np.random.default_rng(2)
    n = 1 << 17
    seqs, count = rng.integers(0, 3, n), rng.integers(0, 4, n)
    first = rng.integers(0, 1 << 30, n) % (np.array(lens)[seqs] - count + 1)
    cu = np.concatenate([[0], np.cumsum(count)])
    k, v = kv.read(c.ints(seqs), c.ints(cu), int(cu[-1]), first=c.ints(first))
    pos = np.arange(cu[-1]) - np.repeat(cu[:-1], count) + np.repeat(first, count)
    start = np.cumsum([0, *lens])[:3]
    where = np.repeat(start[seqs], count) + pos
    at = torch.from_numpy(np.concatenate([c.slots(i, 0, x) for i, x in enumerate(lens)])).cuda()
    for got, x in ((k, c.k[at]), (v, c.v[at])):
        same(got, (held(f64(x), "bfloat16") if bits == 4 else f64(x))[where])
    kv.check()
