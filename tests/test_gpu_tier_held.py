"""Nodes of a tier that are held back until each has a task: equal nodes share them, whatever the speed of host and device, and every
node's result has the lone stage's bits."""
import pytest

from tests.helpers import make_gpu_stage, to_dev
from tests.test_gpu_mfma_parity import SHAPE_G2
from tests.test_gpu_tier import _tier
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,sigma", [(synth.TINY, 0.02), (SHAPE_G2, 0.05)])
def test_queued_work_spreads_and_any_node_gives_the_lone_stage_result(shape, sigma):
    import torch
    S, steps, n_tasks = 48, 5, 9
    layers = [synth.layer_weights(shape, l, 5170, sigma=sigma) for l in range(2)]
    tier = _tier(shape, layers, 3, S + steps + 1, S)
    xs = [to_dev(synth.hidden_states(S, shape, 5180 + q), shape.dtype) for q in range(n_tasks)]
    # 0.2 s ahead of each node's first task, a hundred times what queueing one for each takes (a node's second would wait on the host for the
    # first one's lengths to be read)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(2):  # the first one loads the kernel
        begin.record()
        torch.cuda._sleep(1 << 20)
        end.record()
        end.synchronize()
    cycles = int((1 << 20) * 200.0 / begin.elapsed_time(end))
    for stream in tier.streams:
        with torch.cuda.stream(stream):
            torch.cuda._sleep(cycles)
    tasks = [tier.submit(x, [S], steps, work=1000.0) for x in xs]
    torch.cuda.synchronize()
    assert [t.node for t in tasks[:3]] == [0, 1, 2]
    lone = make_gpu_stage(shape, layers, 1, S + steps + 1, S)
    for x, t in zip(xs, tasks):
        h = lone.prefill(x, [S])[-1:].contiguous()
        for _ in range(steps):
            h = lone.decode_step(h)
        assert torch.equal(h, t.out)
    lone.destroy()
    tier.destroy()
