"""Memory of the cache and its plans where work on it is still to come: on other streams, in graphs."""
import gc

import pytest

from tests.test_gpu_kv_attend import Case

pytestmark = pytest.mark.gpu


def others_like(torch, x, n=6):
    """New tensors that the allocator might put where one of that shape and type was."""
    return [torch.empty(x.shape, dtype=x.dtype, device="cuda") for _ in range(n)]


def test_a_plan_that_a_graph_reads_outlives_its_object():
    c = Case([900, 40, 333], [1, 3, 2])
    torch = c.torch
    want = c.run()
    plan = c.kv.plan(c.seqs, c.cu, c.n_q, heads=c.q.shape[1])
    buffer, cu = plan._buffer, c.cu.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out, lse = c.kv.attend(c.q, plan)
    held, at = torch.empty_like(buffer, device="cpu"), buffer.data_ptr()
    held.copy_(buffer)
    del plan, buffer
    gc.collect()
    new = others_like(torch, held) + [c.kv.plan(c.seqs, c.cu, c.n_q, heads=c.q.shape[1])._buffer for _ in range(3)]
    assert all(not (x.data_ptr() <= at < x.data_ptr() + x.numel()) for x in new)
    for x in new:
        x.fill_(255)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert all((x == 255).all() for x in new) and torch.equal(cu, c.cu)
    c.kv.check()


@pytest.mark.parametrize("explicit", [False, True])
def test_a_plan_that_another_stream_reads_outlives_its_object(explicit):
    c = Case([700, 40, 333], [1, 3, 2])
    torch = c.torch
    want = c.run()
    c.kv._spare.clear()
    seqs, cu = c.seqs.clone(), c.cu.clone()
    plan = c.kv.plan(seqs, cu, c.n_q, heads=c.q.shape[1])
    at = [x.data_ptr() for x in (plan._buffer, seqs, cu)]
    like = [torch.empty_like(x, device="cpu") for x in (plan._buffer, seqs, cu)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # a tenth of a second: what comes now is still to be done below
    if explicit:
        out, lse = c.kv.attend(c.q, plan, stream=side.cuda_stream)
    else:
        with torch.cuda.stream(side):
            out, lse = c.kv.attend(c.q, plan)
    del plan, seqs, cu
    gc.collect()
    for x, old in zip(like, at):
        for y in others_like(torch, x):
            assert y.data_ptr() != old
    assert not side.query()  # the above was in time
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    c.kv.check()


def life(torch, kv, x, **on):
    """Every call that takes lists or values, on 40 sequences of one token."""
    slots = kv.extend(x["seqs"], x["cu"], 40, **on)
    kv.write(slots, x["k"], x["v"], **on)
    kv.attend(x["q"], kv.plan(x["seqs"], x["cu"], 40, heads=2, **on), out=x["out"], lse=x["lse"], **on)
    kv.fork(x["src"], x["dst"], x["tokens"], **on)
    kv.free(x["some"], x["keep"], **on)


def things(torch):
    from paper_2508_14544_gb300 import KVCache
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v, q, out = (torch.randn(40, 2, 16, device="cuda").bfloat16() for _ in range(4))
    return KVCache(64, 16, 2, 16, 41, 8), dict(seqs=ints(range(40)), cu=ints(range(41)), k=k, v=v, q=q, out=out, lse=torch.empty(40, 2, device="cuda"), src=ints([3]),
                                               dst=ints([40]), tokens=ints([1]), some=ints([5]), keep=ints([0]))


@pytest.mark.parametrize("explicit", [False, True])
def test_a_cache_that_another_stream_uses_outlives_its_object(explicit):
    import torch
    life(torch, *things(torch))  # kernels that are loaded at their first launch wait for the GPU
    kv, x = things(torch)
    held = [kv.pool, kv.table, kv.length, kv.ref, kv.status, kv._scratch]
    like, at = [torch.empty_like(y, device="cpu") for y in held], [y.data_ptr() for y in held]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    if explicit:
        life(torch, kv, x, stream=side.cuda_stream)
    else:
        with torch.cuda.stream(side):
            life(torch, kv, x)
    del kv, held
    gc.collect()
    assert all(z.data_ptr() != old for y, old in zip(like, at) for z in others_like(torch, y))
    assert not side.query()  # the above was in time
    side.synchronize()
    assert torch.equal(x["out"], x["v"])  # sequences of one token: its value


def test_tensors_given_to_a_call_on_a_stream_may_be_dropped():
    import torch
    life(torch, *things(torch))
    kv, x = things(torch)
    want = x["v"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    life(torch, kv, x, stream=side.cuda_stream)
    out = x.pop("out")
    like, at = [torch.empty_like(y, device="cpu") for y in x.values()], [y.data_ptr() for y in x.values()]
    x.clear()
    gc.collect()
    assert all(z.data_ptr() != old for y, old in zip(like, at) for z in others_like(torch, y))
    assert not side.query()
    side.synchronize()
    assert torch.equal(out, want)
    assert kv.length.tolist() == [1] * 5 + [0] + [1] * 35
    kv.check()


@pytest.mark.parametrize("how", ["current", "named", "graph"])
def test_a_check_sees_calls_on_other_streams(how):
    import torch

    from paper_2508_14544_gb300 import SimError
    kv, x = things(torch)
    life(torch, kv, x)
    kv.check()
    wrong = torch.tensor([77], dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    if how == "graph":
        with torch.cuda.graph(graph):
            kv.free(wrong)
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        if how == "current":
            kv.free(wrong)
        elif how == "graph":
            graph.replay()
    if how == "named":
        kv.free(wrong, stream=side.cuda_stream)
    with pytest.raises(SimError) as e:
        kv.check()
    assert e.value.code == -1
    kv.check()
