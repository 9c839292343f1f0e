"""What the calls on a 4-bit cache refuse on the host, without a GPU, and the sizes that they give."""
import ctypes

import pytest

from tests.test_kv_refusals import BAD_ARRAYS, BAD_SIZES, INVAL, L, batch, cache  # noqa: F401

BF16_4BIT, F16_4BIT = 16, 17


def read(L, kv, layer=0, n=1, seqs=1 << 24, cu=1 << 24, total=1, k=1 << 24, v=1 << 24, strides=(128, 64, 128, 64)):
    x = lambda p: ctypes.c_void_p(p)  # noqa: E731
    return L.lib().sim_kv_read(ctypes.byref(kv) if kv else None, layer, n, x(seqs), x(cu), None, total, x(k), strides[0], strides[1], x(v), strides[2],
                               strides[3], None)


@pytest.mark.parametrize("dtype", [BF16_4BIT, F16_4BIT])
def test_bad_caches(L, dtype):
    for over in BAD_SIZES[1:] + BAD_ARRAYS:
        kv = cache(L, **{"dtype": dtype, **over})
        x = ctypes.c_void_p(1 << 24)
        assert L.lib().sim_kv_write(ctypes.byref(kv), 0, 1, x, x, 128, 64, x, 128, 64, None) == INVAL, over
        assert read(L, kv) == INVAL, over
        assert L.sim_last_error(None).startswith("sim_kv_read"), L.sim_last_error(None)
        if over in BAD_SIZES:
            assert L.lib().sim_kv_pool_bytes(ctypes.byref(kv)) == 0
    assert read(L, None) == INVAL


@pytest.mark.parametrize("dtype", [2, 3, 15, 18, 32, -1])
def test_types_that_there_are_not(L, dtype):
    kv = cache(L, dtype=dtype)
    assert read(L, kv) == INVAL and L.lib().sim_kv_scratch_bytes(ctypes.byref(kv)) == 0


@pytest.mark.parametrize("dtype", [0, 1, BF16_4BIT, F16_4BIT])
def test_bad_reads(L, dtype):
    kv = cache(L, dtype=dtype)
    for bad in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=(1 << 17) + 1), dict(total=-1), dict(seqs=None), dict(cu=None), dict(k=None), dict(v=None),
                dict(k=(1 << 24) + 8), dict(v=(1 << 24) + 2), *(dict(strides=tuple(4 if i == j else 64 for i in range(4))) for j in range(4))):
        assert read(L, kv, **bad) == INVAL, bad
    assert read(L, kv, n=0, total=0, seqs=None) == 0  # nothing to do


@pytest.mark.parametrize("dim", [8, 32, 40, 64, 80, 96, 104, 128])
def test_sizes(L, dim):
    lib = L.lib()
    for dtype, token in ((0, 2 * dim), (1, 2 * dim), (BF16_4BIT, 20 * -(-dim // 32)), (F16_4BIT, 20 * -(-dim // 32))):
        kv = cache(L, dtype=dtype, head_dim=dim, n_pages=10, n_layers=3, n_kv_heads=5, page_size=32)
        assert lib.sim_kv_pool_bytes(ctypes.byref(kv)) == 10 * 3 * 2 * 5 * 32 * token
        b = batch(L, q_heads=10)
        assert lib.sim_kv_plan_bytes(ctypes.byref(kv), ctypes.byref(b)) > 0 and lib.sim_kv_workspace_bytes(ctypes.byref(kv), ctypes.byref(b)) > 0


def test_bits_that_there_are_not():
    from paper_2508_14544_gb300 import KVCache
    for bits in (0, 2, 8, 32):
        with pytest.raises(ValueError, match="bits"):
            KVCache(8, 16, 2, 64, 4, 4, bits=bits, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        KVCache(8, 16, 2, 64, 4, 4, bits=4, device="cpu")
