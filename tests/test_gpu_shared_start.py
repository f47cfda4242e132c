"""Requests that start with nothing but the shared text: their first token is the one behind it."""
import pytest
import torch

from tests.helpers import to_dev
from tests.test_gpu_shared import SHAPE_BF, _blocks
from workloads import synth

pytestmark = pytest.mark.gpu


# the same sums in another order: a row among several, or alone (test_gpu_shared.py derives the bounds)
@pytest.mark.parametrize("shape,bound", [(synth.TINY, 4e-5), (SHAPE_BF, 1.3e-2)])
def test_a_first_token_is_a_prompt_of_one(shape, bound):
    P, n, seed = 41, 3, 91
    prefix = to_dev(synth.hidden_states(P, shape, seed), shape.dtype)
    *_, blocks = _blocks(shape, 2, seed, prefix, n, budget=8, room=4, sink=1, recent=2)
    x, y = (to_dev(synth.hidden_states(n, shape, seed + i), shape.dtype) for i in (1, 2))
    got = blocks.decode_step(x), blocks.decode_step(y)
    want = blocks.prefill(x, [1] * n), blocks.decode_step(y)
    for a, b in zip(got, want):
        error = float((a.double() - b.double()).norm() / b.double().norm())
        assert error <= bound
