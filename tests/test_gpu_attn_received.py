"""The weight that keys receive (attn_received): how exactly the rows' log-sum-exps count, and the form that calls of many keys take, over the layouts,
rules and masks that the other form's tests have."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import attn_received_cases as cases
from tests.test_gpu_attn import BF, F32, Problem, check_prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rule", [dict(), dict(cap=30.0), dict(slopes=True)])
@pytest.mark.parametrize("held,rows", [(64, 1), (40, 3)])
def test_a_log_sum_exp_counts_in_full(dtype, rule, held, rows):
    """Scores of exactly 0 and a log-sum-exp of z give each seen key e^-z a row.  As an exponent of two, z log2(e) has seven bits before
    the point and is off by up to 2^-18; a weight that carries that is off by up to 2^-18 ln 2 = 2.6e-6 of itself.  What may be off: the exponential
    by 2 units in the last place (2^-22), the remainder of the product (a product of two remainders, below 2^-40) and its factor
    (2^-23), the sums of up to 3 rows (2^-23)."""
    g = torch.Generator().manual_seed(3)
    k = torch.randn((1, 1, held, 64), generator=g).to(dtype).cuda()
    cache = hyp.AttnCache(k, k, torch.tensor([held], dtype=torch.int32, device="cuda"))
    slopes = torch.zeros(1, device="cuda") if rule.get("slopes") else None
    q, start = torch.zeros((rows, 1, 64), dtype=dtype, device="cuda"), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    worst = 0.0
    for z in torch.linspace(44.5, 80.0, 60).tolist():
        lse = torch.full((rows, 1), z, device="cuda")
        exact = math.exp(-float(lse[0, 0].double()))
        got = hyp.attn_received(cache, hyp.AttnRule(0.125, cap=rule.get("cap", 0.0), slopes=slopes), q, start, lse, torch.zeros((1, 1, held), device="cuda"))
        want = torch.tensor([exact * sum(j <= held - rows + i for i in range(rows)) for j in range(held)], dtype=torch.float64)
        worst = max(worst, float(((got[0, 0].double().cpu() - want) / want).abs().max()))
    assert worst <= 2.0 ** -22 + 2.0 ** -40 + 2 * 2.0 ** -23, worst


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", cases.ALL, ids=cases.name)
def test_pairs_of_blocks(dtype, case):
    check_prompt(cases.problem(case, dtype, Problem), last=case["last"])


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d", [128, 33])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_pairs_of_blocks_with_numbers_that_a_row_does_not_see(dtype, d, bad):
    # keys of an id that no row has, beside the others; and behind the requests' last keys, as always
    pr = cases.problem(cases.case(d=d, rule=dict(docs=3)), dtype, Problem)
    pr.q_doc.clamp_(0, 2)
    pr.key_doc[:, :, 7] = pr.key_doc[:, :, 130] = 99
    pr.k[:, :, 7] = pr.k[:, :, 130] = bad
    check_prompt(pr)
