"""Contexts that a stage on a stream of its own hands over, with work before and behind the copies on both streams."""
import pytest
import torch

from tests.helpers import make_gpu_stage, to_dev
from workloads import synth

pytestmark = pytest.mark.gpu


def busy(x):
    for _ in range(40):
        x = (x @ x).clamp(-1, 1)
    return x


def test_contexts_of_a_stage_that_is_at_work_on_its_own_stream():
    from paper_2511_14450_amd import longctx, shared
    shape, lens, n_layers = synth.TINY, [33, 1, 64], 2
    layers = [synth.layer_weights(shape, l, 3, sigma=0.05) for l in range(n_layers)]
    dev = [{k: to_dev(v, shape.dtype) for k, v in w.items()} for w in layers]
    x = to_dev(synth.hidden_states(sum(lens), shape, 50), shape.dtype)
    want, got = (longctx.LongBlocks(shape, dev, 3, most=70, v_format="e2m1") for _ in range(2))
    still = make_gpu_stage(shape, layers, 3, 80, sum(lens))
    still.prefill(x, lens)
    torch.cuda.synchronize()
    want.adopt(still, 0, n_layers)
    prefix = shared.shared_prefix(still, 0, n_layers, request=2)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        stage = make_gpu_stage(shape, layers, 3, 80, sum(lens))
    big = [torch.rand((4096, 4096), device="cuda") for _ in range(2)]
    size = sum(lens) * shape.n_kv_heads * shape.head_dim
    held = torch.full((64, size), 3.0, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        got.reset()
        with torch.cuda.stream(stream):  # the stage's contexts come late on its stream
            busy(big[0])
            stage.prefill(x, lens)
        got.adopt(stage, 0, n_layers)
        for a, b in zip(got.caches, want.caches):
            for s, t in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
                assert torch.equal(s, t)
        with torch.cuda.stream(stream):
            busy(big[0])
            stage.prefill(x, lens)
        for a, b in zip(shared.shared_prefix(stage, 0, n_layers, request=2), prefix):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        torch.cuda.synchronize()
        # memory that the current stream still reads late goes to what is exported
        rows = [held[i].clone() for i in range(64)]
        busy(big[1])
        sums = [r.sum() for r in rows]
        del rows
        got.adopt(stage, 0, n_layers)
        assert all(float(s) == 3.0 * size for s in sums)
    torch.cuda.synchronize()
    stage.destroy()
    still.destroy()
