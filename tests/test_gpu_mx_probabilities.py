"""mx_token beside bf16 rows: what a probability keeps of its bits before it multiplies values, where sums of large terms are small."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import mx_reference as ref
from tests.mx_problem import BF, Problem

pytestmark = pytest.mark.gpu


def bound(out, out_abs, delta):
    """Two bf16 hold a probability to 2^-8 of what the first leaves out of it, 2^-8 at most, so to 2^-16 of itself; it is off by delta, sums by
    2^-19 (mx_reference.out_bound), and the result is rounded once, by at most 2^-8 of itself."""
    return (2 * delta + 2.0 ** -19 + 2.0 ** -16) * out_abs + 2.0 ** -8 * out.abs() + 1e-30


def check(pr, q, scale, blocks=None):
    listed = None if blocks is None else torch.tensor(blocks, dtype=torch.int32).cuda()
    out = hyp.mx_token(pr.cache, hyp.AttnRule(scale), q.cuda(), blocks=listed)[0].double().cpu()
    k, v = pr.values()
    group = q.shape[1] // pr.nkv
    for b, held in enumerate(pr.held):
        for h in range(q.shape[1]):
            c = h // group
            at = list(range(held)) if blocks is None else [j for i in blocks[b][c] if i >= 0 for j in range(i * pr.block, min((i + 1) * pr.block, held))]
            o, _, o_abs, delta = ref.attend(q[b, h], k[b][:, c], v[b][:, c], at, scale=scale)
            assert bool(((out[b, h] - o).abs() <= bound(o, o_abs, delta)).all()), (b, h)


@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e4m3"), ("e2m1", "e2m1")])
@pytest.mark.parametrize("heads,most", [(1, None), (17, None), (24, 70000)])  # the last by two tiles of heads a wave, in parts
@pytest.mark.parametrize("d", [32, 128])
def test_values_that_cancel_leave_what_the_probabilities_differ_by(d, heads, most, formats):
    # keys of probability 1 and values of 1 alternate with keys of 0.5 (1 + x) and values of -2: of each pair -x is left, which is less than half a
    # step of a bf16 beside 0.5
    held = [64, 1000, 3000] + ([5, 300, 1, 0, 32] if most else [])
    pr = Problem(31, held, nkv=1, d=d, formats=formats, dtype=BF, block=0, layout="pages", page=1024, most=most)
    for b, n in enumerate(held):
        odd = (torch.arange(n) % 2).to(BF)
        pr.rows_k[b] = torch.zeros((n, 1, d), dtype=BF)
        pr.rows_k[b][:, 0, 0] = odd
        pr.rows_v[b] = (1 - 3 * odd)[:, None, None].expand(n, 1, d).contiguous()
    pr.fill()
    q = torch.zeros((len(held), heads, d), dtype=BF)
    q[:, :, 0] = -1.0
    for x in (0.9 * 2.0 ** -8, 0.4 * 2.0 ** -8, -0.4 * 2.0 ** -8):
        check(pr, q, math.log(2.0) - math.log1p(x))


@pytest.mark.parametrize("d,heads", [(64, 4), (96, 6), (160, 2), (256, 16)])
def test_rows_of_every_size_within_the_roundings_of_their_results(d, heads):
    pr = Problem(32, [700, 65, 1, 0], nkv=2, d=d, formats=("e4m3", "e4m3"), dtype=BF, block=16).fill()
    q = (torch.randn((4, heads, d), generator=pr.gen) * 1.5).to(BF)
    check(pr, q, d ** -0.5)
    check(pr, q, d ** -0.5, [[[0, 7, 43, -1], [1, 2, -1, 30]], [[4, -1, -1, -1], [0, 1, 2, 3]], [[0, -1, -1, -1], [-1, -1, -1, -1]], [[-1] * 4, [-1] * 4]])
