"""Forms of the operators of hyp_attn.h that a call's size chooses: more requests than a wave has lanes, eviction in one launch and in
several; and infinities and NaN that a row does see, next to those it does not."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests.test_gpu_attn import BF, F32, INF, NAN, Problem, check_prompt, check_token, close
from tests.test_gpu_attn_evict import check as check_evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nkv", [(2, 1), (6, 2)])
@pytest.mark.parametrize("n", [63, 64, 65, 130])
def test_prompts_of_many_requests(n, nq, nkv):
    # with no rows, some, and more than a tile of 128
    held = [(7 * b) % 11 for b in range(n)]
    held[n // 2] = held[n - 1] = 150
    rows = [min(h, b % 3) for b, h in enumerate(held)]
    rows[n // 2] = rows[n - 1] = 140
    check_prompt(Problem(n + nq, BF, nq, nkv, 64, held=held, rows=rows, prefix=5), last=2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nq,nkv", [(1, 1), (6, 2)])
def test_tokens_of_many_requests(dtype, nq, nkv):
    check_token(Problem(nq, dtype, nq, nkv, 64, held=[(13 * b) % 41 for b in range(70)], prefix=140))


@pytest.mark.parametrize("most", [1, 2, 511, 512, 513])
@pytest.mark.parametrize("totals", ["heavy", "ties", "odd"])
def test_eviction_around_the_length_of_one_launch(most, totals):
    held = [most, most // 2, most - 1, 0]
    for keep in {1, (most + 1) // 2, most}:
        check_evict(BF, held, 2, 64, keep, recent=min(keep, 3), totals=totals, room=most)
    check_evict(F32, held, 1, 33, (most + 1) // 2, totals=totals, room=most, page=64, pos=True, doc=True, prefix=9)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 33])
def test_values_that_are_not_finite_and_seen(dtype, d):
    # a feature each of NaN, an infinity, both infinities and a NaN that comes late; the other features of the rows are as before
    pr = Problem(d, dtype, 4, 2, d, held=[90, 140], rows=[90, 70], prefix=20)
    bad = {1: [(10, NAN)], 7: [(40, INF)], 20: [(3, INF), (60, -INF)], 32: [(85, NAN)]}
    finite = pr.v.clone()
    for f, places in bad.items():
        for key, value in places:
            pr.v[:, :, key, f] = value
    q, start, *_ = pr.device()
    out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    pr.v = finite
    want, w_lse, _, bound, b_lse, _ = pr.reference()
    own = torch.tensor(list(range(90)) + list(range(70, 140)))
    for f, places in bad.items():
        for i in range(160):
            seen = [value for key, value in places if key <= own[i]]
            if seen:
                want[i, :, f] = NAN if len(set(seen)) > 1 or math.isnan(seen[0]) else seen[0]
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    clear = ~torch.isnan(want)
    close(out[clear.cuda()], want[clear], bound[clear], "out")
    close(lse, w_lse, b_lse, "lse")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", ["q", "k", "v", "prefix"])
def test_all_nan(dtype, what):
    pr = Problem(3, dtype, 4, 2, 64, held=[200, 130], rows=[200, 30], prefix=40)
    for t in {"q": (pr.q,), "k": (pr.k,), "v": (pr.v,), "prefix": (pr.pk, pr.pv)}[what]:
        t.fill_(NAN)
    q, start, *_ = pr.device()
    out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all()) == (what != "v")
    out, _ = hyp.attn_token(pr.cache, pr.rule, q[:2].contiguous())
    assert bool(torch.isnan(out).all())


def test_parts_whose_sums_are_lost_meet_parts_that_are_not():
    # one row over many keys is cut into parts; a NaN score in one of them, whose other weights are nothing next to the others'
    pr = Problem(4, F32, 2, 1, 64, held=[3000], prefix=0)
    pr.q[:] = 0.0
    pr.q[..., 0] = 8.0
    pr.k[..., 0] = torch.where(torch.arange(pr.k.shape[2]) < 1500, -400.0, 400.0)
    pr.k[0, 0, 100, 1] = NAN
    q, *_ = pr.device()
    out, lse = hyp.attn_token(pr.cache, pr.rule, q)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("most", [255, 256, 257])
def test_eviction_in_one_launch_and_in_two(most):
    for totals in ("heavy", "ties", "odd"):
        check_evict(BF, [most, most // 2, most - 1, 0], 2, 64, (most + 1) // 2, recent=3, totals=totals, room=most)
        check_evict(F32, [most, 3], 1, 33, most - 2, totals=totals, room=most, page=64, pos=True, doc=True, prefix=9)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 2, 4, 5, 8, 9])
def test_rows_at_the_shared_keys_around_a_wave(dtype, n):
    check_token(Problem(n, dtype, 4, 1, 64, held=[5 + 9 * b for b in range(n)], prefix=300))


def test_received_weight_by_pairs_of_blocks_and_by_blocks():
    # 160 pairs of blocks: the weight of many prompts of one key head, and of one less
    for n in (160, 159):
        held = [(17 * b) % 40 + 1 for b in range(n)]
        held[3] = 140
        check_prompt(Problem(n, BF, 5, 1, 40, held=held, rows=[min(h, 30) for h in held]), last=0)
