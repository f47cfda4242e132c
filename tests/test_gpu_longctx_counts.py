"""What blocks over long contexts hold after a call that is refused or fails: as many keys as before, or none where the old ones are lost."""
import dataclasses

import pytest
import torch

from tests.helpers import make_gpu_stage, to_dev
from workloads import synth

pytestmark = pytest.mark.gpu
LENS = [20, 1, 9]


def rows(shape, n, seed):
    return to_dev(synth.hidden_states(n, shape, seed), shape.dtype)


@pytest.fixture
def made():
    from paper_2511_14450_amd import longctx
    shape = synth.TINY
    layers = [synth.layer_weights(shape, l, 3, sigma=0.05) for l in range(2)]
    dev = [{k: to_dev(v, shape.dtype) for k, v in w.items()} for w in layers]
    blocks, same = (longctx.LongBlocks(shape, dev, 3, 40, read_blocks=2, block_keys=16, sink=0, recent=1) for _ in range(2))
    for b in (blocks, same):
        b.prefill(rows(shape, sum(LENS), 1), LENS)
    return shape, layers, blocks, same


def as_before(shape, blocks, same):
    assert blocks.held == LENS and blocks.lens.tolist() == LENS
    x = rows(shape, 3, 2)
    assert torch.equal(blocks.decode_step(x), same.decode_step(x))


def test_a_refused_adoption_drops_nothing(made):
    shape, layers, blocks, same = made
    long = make_gpu_stage(shape, layers, 3, 80, 80)
    long.prefill(rows(shape, 50, 3), [41, 4, 5])
    with pytest.raises(ValueError, match="more than 40"):
        blocks.adopt(long, 0, 2)
    for l_start, l_end in ((-1, 1), (1, 3), (0, 1)):
        with pytest.raises(ValueError, match="blocks"):
            blocks.adopt(long, l_start, l_end)
    few = make_gpu_stage(shape, layers, 3, 80, 80)
    few.prefill(rows(shape, 5, 4), [2, 3])
    with pytest.raises(RuntimeError, match="no such request"):
        blocks.adopt(few, 0, 2)
    # the same width of keys in heads of another size
    other = dataclasses.replace(shape, n_q_heads=2 * shape.n_q_heads, n_kv_heads=2 * shape.n_kv_heads, head_dim=shape.head_dim // 2)
    split = make_gpu_stage(other, layers, 3, 80, 80)
    split.prefill(rows(shape, 12, 5), [3, 4, 5])
    with pytest.raises(ValueError, match="KV heads"):
        blocks.adopt(split, 0, 2)
    as_before(shape, blocks, same)
    for stage in (long, few, split):
        stage.destroy()


def test_an_adoption_that_fails_underway_leaves_no_keys(made, monkeypatch):
    shape, layers, blocks, _ = made
    stage = make_gpu_stage(shape, layers, 3, 80, 80)
    stage.prefill(rows(shape, 12, 6), [3, 4, 5])
    export = stage.export_kv

    def fails(layer, request):
        if layer == 1:
            raise MemoryError
        return export(layer, request)

    monkeypatch.setattr(stage, "export_kv", fails)
    with pytest.raises(MemoryError):
        blocks.adopt(stage, 0, 2)
    assert blocks.held == [0] * 3 and blocks.lens.tolist() == [0] * 3
    monkeypatch.undo()
    blocks.adopt(stage, 0, 2)
    assert blocks.held == [3, 4, 5] and blocks.lens.tolist() == [3, 4, 5]
    stage.destroy()


def test_rows_that_do_not_go_through_the_blocks_are_not_counted(made):
    shape, _, blocks, same = made
    for bad in (torch.zeros((3, shape.hidden + 1), device="cuda"), torch.zeros((3, shape.hidden), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, shape.hidden))):
        with pytest.raises((ValueError, RuntimeError)):
            blocks.prefill(bad, [1, 1, 1])
        with pytest.raises((ValueError, RuntimeError)):
            blocks.decode_step(bad)
    as_before(shape, blocks, same)
