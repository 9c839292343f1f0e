"""The cache serves: it has no backward pass, and says so instead of leaving a result without its graph."""
import pytest

pytestmark = pytest.mark.gpu


def test_tensors_that_require_a_gradient_are_refused():
    import torch

    from paper_2508_14544_gb300 import KVCache
    kv = KVCache(4, 16, 2, 16, 2, 2)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs, cu = ints([0]), ints([0, 3])
    slots = kv.extend(seqs, cu, 3)
    k, v, q = (torch.randn(3, 2, 16, device="cuda").bfloat16() for _ in range(3))
    grad = k.clone().requires_grad_()
    for bad in ((grad, v), (k, grad), (grad * 2, v)):
        with pytest.raises(ValueError, match="gradient"):
            kv.write(slots, *bad)
    kv.write(slots, k, v)
    plan = kv.plan(seqs, cu, 3, heads=2)
    for bad in (dict(q=grad), dict(q=q, out=torch.empty_like(q).requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            kv.attend(plan=plan, **bad)
    want = kv.attend(k, plan)
    with torch.no_grad():
        kv.write(slots, grad.detach(), v)
        got = kv.attend(grad, plan)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(kv.attend(grad.detach(), plan)[0], want[0])
    kv.check()
