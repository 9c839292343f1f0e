"""The replay of a schedule: its batches from completions (CPU), and a whole instance on the GPU."""
import numpy as np
import pytest


def test_batches_of_a_schedule():
    from paper_2508_14544_gb300.replay import batches
    # requests 0, 1, 2 run in steps [0, 2), [1, 2) and [5, 6): steps 2..4 are idle
    got = [tuple(x.tolist() for x in b) for b in batches([0, 1, 5], [2, 2, 6])]
    assert got == [([0], [], []), ([1], [0], [0, 1]), ([2], [], [2])]
    assert batches([], []) == []


def test_batches_add_up_to_the_simulated_schedule():
    """Batch sizes and step memories of H-SF on the 50-request instance, from the oracle's completions."""
    from oracle import plain
    from paper_2508_14544_gb300 import POLICIES
    from paper_2508_14544_gb300 import workloads as W
    from paper_2508_14544_gb300.replay import batches
    w = W.make_workload("c1")
    for policy in ("A_max", "H-SF"):
        res, completion = plain.run_workload(POLICIES[policy], w, completions=True)
        start = completion - w.true_o
        steps = batches(start, completion)
        assert len(steps) == res["steps"][0]
        assert sum(len(a) + len(b) for a, b, _ in steps) == res["request_steps"][0]
        assert sum(len(d) for _, _, d in steps) == w.n_total
        length, peak = np.zeros(w.n_total, int), 0
        for new, old, _ in steps:
            length[new] += w.prompt[new] + 1
            length[old] += 1
            peak = max(peak, int(length[new].sum() + length[old].sum()))
        assert peak == res["peak_memory"][0]


def test_a_policy_that_cancels_is_refused():
    from paper_2508_14544_gb300 import workloads as W
    from paper_2508_14544_gb300.replay import run
    with pytest.raises(ValueError):
        run(W.make_workload("c1"), policy="A_min")


@pytest.mark.gpu
@pytest.mark.parametrize("policy,prefix", [("A_max", 0), ("H-SF", 333), ("A_r", 64)])
def test_replay_of_the_50_request_instance(policy, prefix):
    from paper_2508_14544_gb300 import workloads as W
    from paper_2508_14544_gb300.replay import run
    d = run(W.make_workload("c1"), policy=policy, layers=2, group=2, prefix=prefix)
    assert d["steps"] > 50 and d["peak_tokens"] <= 2000 and d["us_per_step"] > 0
    assert np.isfinite(d["coef_us"]).all() and np.isfinite(d["total_latency_us"]) and d["makespan_us"] > 0
