"""Rules at the end of the range of a float."""
import pytest
import torch

import paper_2511_14450_amd as hyp
from tests.test_gpu_attn import BF, F32, Problem, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap", [1e-30, 1e-38, 1e-41])
def test_a_cap_far_below_the_scale(dtype, cap):
    # every score is a tanh of -1, 0 or 1 times nothing: rows that are zeros have scores of 0, not of 0 * infinity
    pr = Problem(41, dtype, 4, 2, 64, held=[90, 33], rows=[90, 20], prefix=40, cap=cap)
    pr.q[::3] = 0.0
    q, start, *_ = pr.device()
    out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    want, w_lse, w_tot, bound, b_lse, b_tot = pr.reference()
    close(out, want, bound, "out")
    close(lse, w_lse, b_lse, "lse")
    got = hyp.attn_received(pr.cache, pr.rule, q, start, lse, torch.zeros((2, 2, 90), device="cuda"))
    close(got, w_tot, b_tot + 2.0 ** -23 * (1 + w_tot), "totals")
    tok, _ = hyp.attn_token(pr.cache, pr.rule, q[[89, 109]].contiguous())
    close(tok, want[[89, 109]], bound[[89, 109]], "single tokens")
