"""What lies in the pool of a 4-bit cache: lo, step and codes of every group, by the definition."""
import numpy as np
import pytest

from tests.kv_4bit_reference import BITS, held, round16
from tests.test_gpu_kv_4bit import SPECIAL, Pool, f64, special

pytestmark = pytest.mark.gpu


def parts(x, dtype):
    """lo and step [.., groups] and codes [.., D] of finite values x [.., D] in 64 bits; held: lo + code step on the type's grid."""
    lo, step, code = [], [], []
    for a in range(0, x.shape[-1], 32):
        y = x[..., a: a + 32]
        low, high = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
        s = np.where(high > low, np.maximum(round16((high - low) / 15, dtype, down=True), 2.0 ** BITS[dtype][1]), 0.0)
        some = np.where(s > 0, s, 1.0)
        t = y - low  # with rest, exactly
        rest = (y - (t - (t - y))) - (low + (t - y))
        k = np.floor(t / some)
        border = (k + 0.5) * some
        on = (t == border) & (rest == 0)
        lo.append(low)
        step.append(s)
        code.append(np.minimum(k + np.where(on, k % 2, (t > border) | ((t == border) & (rest > 0))), 15))
    return np.concatenate(lo, -1), np.concatenate(step, -1), np.concatenate(code, -1)


def in_pool(c, n):
    """lo, step and codes of sequence 0's n tokens: two arrays each, of the keys and of the values, [tokens, heads, ..]."""
    G, heads, D = -(-c.dim // 32), c.heads, c.dim
    strips = c.kv.pool[:, 0].reshape(-1, 2, heads, c.page // 16, 320 * G).cpu().numpy()
    t = np.arange(n)
    strips = strips[c.table[0, t[::16] // c.page], :, :, t[::16] % c.page // 16]  # [strips, 2, heads, bytes]
    m = len(strips)
    d = np.arange(D)

    def floats(x):
        return (x.astype(np.uint32) << 16).view(np.float32) if c.dtype == "bfloat16" else x.view(np.float16)
    k, v = (np.ascontiguousarray(strips[:, i]) for i in (0, 1))
    words = k[..., : 256 * G].view(np.uint32).reshape(m, heads, 16, 4, G)
    kc = words[..., d % 32 // 8, d // 32] >> (4 * (d % 8 // 2) + 16 * (d % 2)).astype(np.uint32) & 15
    ks = floats(k[..., 256 * G:].view(np.uint16)).reshape(m, heads, 16, G, 2)
    words = v[..., : 256 * G].view(np.uint16).reshape(m, heads, 2, 8, 4, G, 2).transpose(0, 1, 2, 4, 6, 3, 5).reshape(m, heads, 16, 8, G)
    vc = words[..., d % 32 // 4, d // 32] >> (4 * (d % 4)).astype(np.uint16) & 15
    vs = floats(v[..., 256 * G:].view(np.uint16)).reshape(m, heads, 8, G, 2, 2).transpose(0, 1, 2, 5, 3, 4).reshape(m, heads, 16, G, 2)

    def rows(x):
        return x.swapaxes(1, 2).reshape(m * 16, heads, -1)[:n].astype(np.float64)
    return [(rows(s[..., 1]), rows(s[..., 0]), rows(x)) for s, x in ((ks, kc), (vs, vc))]


def same_parts(c, n):
    import torch
    at = torch.from_numpy(c.slots(0, 0, n)).cuda()
    for got, x in zip(in_pool(c, n), (f64(c.k[at]), f64(c.v[at]))):
        want = parts(x, c.dtype)
        wide = np.repeat(want[0], 32, -1)[..., : c.dim] + want[2] * np.repeat(want[1], 32, -1)[..., : c.dim]
        assert np.array_equal(round16(wide, c.dtype), held(x, c.dtype))
        for name, a, b in zip(("lo", "step", "codes"), got, want):
            bad = a != b
            assert not bad.any(), (name, np.argwhere(bad)[:4].tolist(), a[bad][:4], b[bad][:4])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("kind", SPECIAL)
def test_every_group_by_the_definition(kind, dtype):
    import torch
    c = Pool([333], dim=80, page=32, dtype=dtype, make=special(kind, torch, dtype), fill=0)
    same_parts(c, 333)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [128, 32, 72])
def test_groups_of_one_value_have_no_step(dim, dtype):
    """Of every size: from the smallest floats to the largest ones, of both signs."""
    import torch
    n = 400

    def make(n):
        bits = torch.randint(0, 0x7f80 if dtype == "bfloat16" else 0x7c00, (n, 2, -(-dim // 32)), generator=torch.Generator("cuda").manual_seed(dim), device="cuda")
        top = 0x7f7f if dtype == "bfloat16" else 0x7bff
        bits[::5] = top - bits[::5] % 40  # next to the largest
        x = bits.to(torch.int16).view(getattr(torch, dtype))
        x = torch.where((bits % 3 == 0) & (bits > 0), -x, x)
        return x.repeat_interleave(32, -1)[..., :dim]
    c = Pool([n], dim=dim, dtype=dtype, make=make, fill=0)
    same_parts(c, n)
    assert not any(step.any() or code.any() for _, step, code in in_pool(c, n))
