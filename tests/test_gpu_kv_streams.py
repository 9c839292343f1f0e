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
