"""Ids and counts at the end of their range: every negative id sees and is seen by all, -2^31 too, and a count of none shows nothing."""
import pytest
import torch

from tests.test_gpu_attn import BF, F32, Problem, check_prompt, check_token

pytestmark = pytest.mark.gpu
LEAST = -2 ** 31


def documents(dtype, seed, **more):
    pr = Problem(seed, dtype, 4, 2, 64, held=[150, 90], rows=more.pop("rows", [150, 40]), docs=3, **more)
    pr.key_doc[:] = torch.arange(pr.key_doc.shape[2], dtype=torch.int32) // 40
    own = list(range(150)) + list(range(50, 90)) if not pr.token else [149, 89]
    pr.q_doc[:] = torch.tensor([o // 40 for o in own], dtype=torch.int32)
    return pr


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("of", ["a row", "a key", "both", "all rows"])
def test_the_least_id_is_one_that_sees_all(dtype, of):
    pr = documents(dtype, 31)
    if of in ("a row", "both"):
        pr.q_doc[::7] = LEAST  # some of the rows that a wave has, whatever wave it is
    if of in ("a key", "both"):
        pr.key_doc[:, :, 12] = LEAST
    if of == "all rows":
        pr.q_doc[:] = LEAST
    check_prompt(pr)
    tok = documents(dtype, 32, rows=None)
    tok.q_doc[0], tok.key_doc[:, :, 12] = LEAST, LEAST
    check_token(tok)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_least_count_shows_nothing(dtype):
    check_prompt(Problem(33, dtype, 4, 2, 64, held=[150, 90], rows=[150, 40], prefix=10, see_all=[LEAST, LEAST + 1]))
