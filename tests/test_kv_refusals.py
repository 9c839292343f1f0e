"""What the paged cache's C ABI refuses on the host, without a GPU: nothing is launched by a refused call."""
import ctypes

import pytest

INVAL = -1


@pytest.fixture(scope="module")
def L():
    from paper_2508_14544_gb300 import _lib, build
    try:
        build.build()
    except RuntimeError as e:
        pytest.skip(str(e))
    _lib.lib()
    return _lib


def cache(L, **over):
    at = dict(pool=1 << 20, table=2 << 20, length=3 << 20, ref=4 << 20, status=5 << 20, scratch=6 << 20, dtype=0, n_pages=10, n_layers=2, n_kv_heads=2,
              page_size=16, head_dim=64, max_seqs=8, max_pages=4)
    return L.sim_kv(**{**at, **over})


BAD_SIZES = [dict(dtype=2), dict(n_pages=0), dict(n_pages=(1 << 28) + 1), dict(n_layers=0), dict(n_kv_heads=0), dict(page_size=8), dict(page_size=48),
             dict(page_size=256), dict(head_dim=0), dict(head_dim=4), dict(head_dim=100), dict(head_dim=136), dict(max_seqs=0), dict(max_seqs=(1 << 17) + 1),
             dict(max_pages=0), dict(max_pages=1 << 26), dict(n_layers=1 << 16, n_kv_heads=1 << 16)]
BAD_ARRAYS = [dict(pool=None), dict(table=None), dict(length=None), dict(ref=None), dict(status=None), dict(scratch=None), dict(pool=(1 << 20) + 8),
              dict(ref=(4 << 20) + 4), dict(scratch=(6 << 20) + 8)]


def calls(L, kv, b):
    lib, p, x = L.lib(), ctypes.byref(kv) if kv else None, ctypes.c_void_p(1 << 24)
    return {"extend": lambda: lib.sim_kv_extend(p, 1, x, x, 1, x, None), "write": lambda: lib.sim_kv_write(p, 0, 1, x, x, 128, 64, x, 128, 64, None),
            "fork": lambda: lib.sim_kv_fork(p, 1, x, x, None, None), "copy": lambda: lib.sim_kv_copy(p, 1, x, x, None),
            "free": lambda: lib.sim_kv_free(p, 1, x, None, None), "compact": lambda: lib.sim_kv_compact(p, x, None),
            "plan": lambda: lib.sim_kv_plan(p, ctypes.byref(b), None),
            "attend": lambda: lib.sim_kv_attend(p, ctypes.byref(b), 0, x, 128, 64, ctypes.c_float(1.0), x, 128, 64, None, None)}


def batch(L, **over):
    return L.sim_kv_batch(**{**dict(n=2, n_q=2, q_heads=4, n_groups=0, seqs=1 << 20, cu_q=1 << 20, cu_group=None, plan=1 << 20, workspace=1 << 20), **over})


@pytest.mark.parametrize("over", BAD_SIZES + BAD_ARRAYS + [None])
def test_a_bad_cache(L, over):
    kv = cache(L, **over) if over is not None else None
    for name, call in calls(L, kv, batch(L)).items():
        assert call() == INVAL, name
        assert L.sim_last_error(None).startswith("sim_kv_" + name), L.sim_last_error(None)
    if over in BAD_SIZES:
        assert L.lib().sim_kv_scratch_bytes(ctypes.byref(kv)) == 0
        assert L.lib().sim_kv_plan_bytes(ctypes.byref(kv), ctypes.byref(batch(L))) == 0


def test_bad_lists(L):
    lib, p, x = L.lib(), ctypes.byref(cache(L)), ctypes.c_void_p(1 << 24)
    for n in (-1, 9):
        assert lib.sim_kv_extend(p, n, x, x, 1, x, None) == INVAL
        assert lib.sim_kv_fork(p, n, x, x, None, None) == INVAL
        assert lib.sim_kv_copy(p, n, x, x, None) == INVAL
        assert lib.sim_kv_free(p, n, x, None, None) == INVAL
    assert lib.sim_kv_extend(p, 1, None, x, 1, x, None) == INVAL
    assert lib.sim_kv_extend(p, 1, x, None, 1, x, None) == INVAL
    assert lib.sim_kv_extend(p, 1, x, x, 1, None, None) == INVAL
    assert lib.sim_kv_extend(p, 1, x, x, -1, x, None) == INVAL
    assert lib.sim_kv_fork(p, 1, x, None, None, None) == INVAL
    assert lib.sim_kv_copy(p, 1, None, x, None) == INVAL
    assert lib.sim_kv_free(p, 1, None, None, None) == INVAL
    assert lib.sim_kv_compact(p, None, None) == INVAL
    odd = ctypes.c_void_p((1 << 24) + 1)
    for layer, n, slots, k, v in ((2, 1, x, x, x), (-1, 1, x, x, x), (0, -1, x, x, x), (0, 1, None, x, x), (0, 1, x, None, x), (0, 1, x, x, None),
                                  (0, 1, x, odd, x), (0, 1, x, x, odd)):
        assert lib.sim_kv_write(p, layer, n, slots, k, 128, 64, v, 128, 64, None) == INVAL


@pytest.mark.parametrize("over", [dict(n=-1), dict(n=(1 << 17) + 1), dict(n_q=-1), dict(n_q=1 << 29), dict(q_heads=0), dict(q_heads=3), dict(n_groups=-1),
                                  dict(n_groups=3, cu_group=1 << 20), dict(n_groups=1), dict(seqs=None), dict(cu_q=None), dict(plan=None),
                                  dict(workspace=None), dict(plan=(1 << 20) + 8), dict(workspace=(1 << 20) + 4)])
def test_a_bad_batch(L, over):
    c = calls(L, cache(L), batch(L, **over))
    assert c["plan"]() == INVAL and c["attend"]() == INVAL


def test_sizes_whose_products_are_too_large(L):
    kv = cache(L, n_kv_heads=1 << 10, max_pages=1 << 23)  # 2^27 tokens for each of 2^10 heads
    assert L.lib().sim_kv_scratch_bytes(ctypes.byref(kv)) == 0
    kv = cache(L, n_kv_heads=1 << 10, max_seqs=1 << 17)
    assert L.lib().sim_kv_scratch_bytes(ctypes.byref(kv)) > 0
    for n, ok in ((1 << 16, True), ((1 << 16) + 1, False)):
        assert (L.lib().sim_kv_plan_bytes(ctypes.byref(kv), ctypes.byref(batch(L, n=n, q_heads=1 << 10))) > 0) is ok


def test_a_scale_that_overflows_as_a_power_of_two(L):
    """exp(s x) is computed as 2^(s log2(e) x): that product has to be finite too."""
    lib, p, b, x = L.lib(), ctypes.byref(cache(L)), ctypes.byref(batch(L)), ctypes.c_void_p(1 << 24)
    assert lib.sim_kv_attend(p, b, 0, x, 128, 64, ctypes.c_float(3e38), x, 128, 64, None, None) == INVAL


def test_bad_attention_arguments(L):
    lib, p, b, x = L.lib(), ctypes.byref(cache(L)), ctypes.byref(batch(L)), ctypes.c_void_p(1 << 24)

    def attend(layer=0, q=x, scale=1.0, out=x, ot=128, oh=64):
        return lib.sim_kv_attend(p, b, layer, q, 128, 64, ctypes.c_float(scale), out, ot, oh, None, None)
    for bad in (dict(layer=-1), dict(layer=2), dict(q=None), dict(q=ctypes.c_void_p((1 << 24) + 1)), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(out=None), dict(out=ctypes.c_void_p((1 << 24) + 8)), dict(ot=132), dict(oh=68)):
        assert attend(**bad) == INVAL, bad


def test_empty_calls_do_nothing(L):
    lib, p, x = L.lib(), ctypes.byref(cache(L)), ctypes.c_void_p(1 << 24)
    assert lib.sim_kv_extend(p, 0, None, None, 0, None, None) == 0
    assert lib.sim_kv_write(p, 0, 0, None, None, 0, 0, None, 0, 0, None) == 0
    assert lib.sim_kv_fork(p, 0, None, None, None, None) == 0
    assert lib.sim_kv_copy(p, 0, None, None, None) == 0
    assert lib.sim_kv_free(p, 0, None, None, None) == 0
    assert lib.sim_kv_attend(p, ctypes.byref(batch(L, n_q=0)), 0, x, 128, 64, ctypes.c_float(1.0), x, 128, 64, None, None) == 0


def test_python_refuses_other_tensors():
    import torch

    from paper_2508_14544_gb300 import KVCache
    good = dict(pool=torch.zeros(4, 1, 2, 2, 16, 64, dtype=torch.bfloat16), table=torch.zeros(3, 4, dtype=torch.int32),
                length=torch.zeros(3, dtype=torch.int32), ref=torch.zeros(4, dtype=torch.int32))
    for name, x in (("pool", torch.zeros(4, 1, 2, 2, 16, 64)), ("pool", good["pool"]), ("pool", torch.zeros(4, 2, 16, 64, dtype=torch.float16)),
                    ("table", torch.zeros(3, 4)), ("length", torch.zeros(4, dtype=torch.int32)), ("ref", torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            KVCache.wrap(**{**good, name: x})


def test_tokens_without_entries_need_their_offsets(L):
    """n_new slots are to be written, as of no entry: not without the one offset that there is."""
    lib, p, x = L.lib(), ctypes.byref(cache(L)), ctypes.c_void_p(1 << 24)
    assert lib.sim_kv_extend(p, 0, None, None, 3, x, None) == INVAL
    assert L.sim_last_error(None).startswith("sim_kv_extend")
