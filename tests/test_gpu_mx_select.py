"""mx_select against its definition: ties, NaN, always kept blocks, both launch forms, groups of every size."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import mx_reference as ref
from tests.mx_problem import BF, F32, Problem

pytestmark = pytest.mark.gpu


def bare(seed, held, nkv, d, block, layout="slab", quant=None, page=None):
    """A cache whose bounds are drawn, not written"""
    pr = Problem(seed, held, nkv=nkv, d=d, block=block, layout=layout, page=page or max(32, 2 * block), formats=("e2m1", "e2m1"))
    mid, wide = (torch.randn(pr.lo.shape, generator=pr.gen) for _ in range(2))
    if quant:
        mid, wide = (mid * quant).round() / quant, (wide * quant).round() / quant
    pr.lo.copy_(mid - wide.abs())
    pr.hi.copy_(mid + wide.abs())
    pr.lens.copy_(torch.tensor(held, dtype=torch.int32))
    return pr


def want(pr, q, keep, sink, recent):
    lo, hi, group, out = pr.lo.float().cpu(), pr.hi.float().cpu(), q.shape[1] // pr.nkv, []
    for b, held in enumerate(pr.held):
        held = min(max(held, 0), pr.most)
        for c in range(pr.nkv):
            at = [pr.place(b, i, pr.lo.shape[2]) for i in range(-(-held // pr.block))]
            l, h = ([t[page, c, i] for page, i in at] for t in (lo, hi))
            out.append(ref.select(q[b, c * group:(c + 1) * group].float().cpu(), l, h, held, pr.block, keep, sink, recent))
    return torch.tensor(out, dtype=torch.int32).reshape(len(pr.held), pr.nkv, keep)


def check(pr, q, keep, sink=0, recent=0):
    got = hyp.mx_select(pr.cache, q.cuda(), keep, sink=sink, recent=recent)
    assert torch.equal(got.cpu(), want(pr, q, keep, sink, recent))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("group,d", [(1, 64), (4, 128), (5, 80), (3, 200), (9, 33), (4, 256)])
def test_the_best_blocks_of_short_and_long_requests(dtype, group, d):
    # up to 256 blocks in one launch, more in two
    for held, keep in (([900, 16, 0, 4096], 7), ([9000, 100, 4800], 11)):
        pr = bare(1, held, 2, d, 16)
        check(pr, torch.randn((len(held), 2 * group, d), generator=pr.gen).to(dtype), keep, 1, 2)


@pytest.mark.parametrize("layout", ["slab", "pages", "inner"])
@pytest.mark.parametrize("block", [16, 64, 256])
def test_layouts_and_block_sizes(layout, block):
    for held in ([40 * block - 3, block, 7 * block + 1], [300 * block, 280 * block - 5]):
        pr = bare(2, held, 2, 96, block, layout)
        check(pr, torch.randn((len(held), 6, 96), generator=pr.gen), 9, 0, 1)


@pytest.mark.parametrize("blocks", [200, 700, 5000, 9000])
@pytest.mark.parametrize("quant", [1, 8])
def test_equal_scores_go_to_the_first_blocks(blocks, quant):
    # whole numbers, of which many sums are equal; more equal ones than are ranked one by one; requests of more blocks than one look holds
    pr = bare(3, [blocks * 16, blocks * 16 - 40], 1, 8, 16, quant=quant)
    q = torch.randint(-2, 3, (2, 2, 8), generator=pr.gen).float()
    for keep, sink, recent in ((1, 0, 0), (blocks // 3, 0, 0), (blocks - 1, 3, 5), (9, 4, 5), (blocks // 2, blocks // 4, 0)):
        check(pr, q, keep, sink, recent)
    check(pr, torch.zeros((2, 2, 8)), blocks // 2, 1, 1)  # all are equal
    pr.lo.fill_(1.0)
    pr.hi.fill_(1.0)
    check(pr, q, 5, 0, 2)


@pytest.mark.parametrize("blocks", [100, 3000])
def test_nan_infinities_and_signed_zeros(blocks):
    pr = bare(4, [blocks * 16], 1, 16, 16)
    pr.lo[0, 0, 5] = math.nan
    pr.hi[0, 0, 5] = math.nan
    pr.lo[0, 0, 70, 3], pr.hi[0, 0, 70, 3] = math.nan, math.nan
    pr.hi[0, 0, 90] = math.inf
    pr.lo[0, 0, 40:60], pr.hi[0, 0, 40:60] = -0.0, 0.0
    q = torch.randn((1, 2, 16), generator=pr.gen)
    for keep, sink, recent in ((1, 0, 0), (2, 0, 0), (3, 1, 1), (20, 0, 3), (blocks - 2, 0, 0)):
        check(pr, q, keep, sink, recent)
    q[0, 1, 2] = math.nan
    check(pr, q, 4)
    q[0, 0, 2] = -math.inf
    check(pr, q, 4, 0, 1)


def test_scores_that_differ_in_the_last_bits_of_a_float():
    # 2^20 + i * 2^-6 in exact arithmetic: a float holds steps of 2^-3 there
    pr = bare(5, [400 * 16], 1, 4, 16)
    i = torch.randperm(400, generator=pr.gen)
    pr.hi.zero_()
    pr.lo.zero_()
    pr.hi[0, 0, :, 0] = 2.0 ** 20
    pr.hi[0, 0, :, 1] = (i % 16).to(BF).cuda() * 2.0 ** -6
    pr.hi[0, 0, :, 2] = (i // 16).to(BF).cuda() * 2.0 ** -2
    got = hyp.mx_select(pr.cache, torch.ones((1, 1, 4), device="cuda"), 37)
    assert got[0, 0].tolist() == sorted((i >= 363).nonzero()[:, 0].tolist())


def test_a_request_keeps_all_it_has_and_lengths_are_cut():
    pr = bare(6, [5 * 16, 16 * 16, 0], 2, 32, 16)
    q = torch.randn((3, 4, 32), generator=pr.gen)
    check(pr, q, 40)
    assert hyp.mx_select_workspace_bytes(pr.cache, q.cuda(), 40) == 0
    pr.held = [2 ** 31 - 1, -3, 17]
    pr.lens.copy_(torch.tensor(pr.held, dtype=torch.int32))
    check(pr, q, 4, 1, 1)


def test_no_key_of_a_block_passes_its_score():
    pr = Problem(7, [500], nkv=2, d=96, block=32, formats=("e2m1", "e2m1")).fill()
    q = torch.randn((1, 6, 96), generator=pr.gen)
    k = pr.values()[0][0]
    lo, hi = pr.lo.double().cpu()[0], pr.hi.double().cpu()[0]
    for h in range(6):
        row, c = q[0, h].double(), h // 3
        score = (torch.where(row >= 0, hi[c] * row, lo[c] * row)).sum(-1)
        best = torch.stack([part.max() for part in (k[:, c] @ row).split(32)])
        assert bool((best <= score[:16] + 1e-9).all())
    check(pr, q, 5, 1, 1)
