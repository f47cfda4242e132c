"""mx_token against the formula in 64 bits over the numbers that the cache holds."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import mx_reference as ref
from tests.mx_problem import BF, F32, Problem

pytestmark = pytest.mark.gpu


def rows(pr, heads, dtype, sigma=1.5):
    return (torch.randn((len(pr.held), heads, pr.d), generator=pr.gen) * sigma).to(dtype)


def check(pr, q, blocks=None, cap=0.0, slopes=None, scale=None, got=None, values=None):
    """blocks: lists of listed blocks, [request][head]"""
    n, heads, d = q.shape
    scale, group = scale or d ** -0.5, heads // pr.nkv
    if got is None:
        rule = hyp.AttnRule(scale, cap=cap, slopes=None if slopes is None else torch.tensor(slopes).cuda())
        listed = None if blocks is None else torch.tensor(blocks, dtype=torch.int32).cuda()
        got = hyp.mx_token(pr.cache, rule, q.cuda(), blocks=listed)
    out, lse = (t.double().cpu() for t in got)
    k, v = values or pr.values()
    for b, held in enumerate(pr.held):
        for h in range(heads):
            c = h // group
            at = list(range(held)) if blocks is None else [j for i in blocks[b][c] if 0 <= i for j in range(i * pr.block, min((i + 1) * pr.block, held))]
            o, z, o_abs, delta = ref.attend(q[b, h], k[b][:, c], v[b][:, c], at, scale=scale, cap=cap, slope=slopes[h] if slopes else 0.0, length=held)
            assert bool(((out[b, h] - o).abs() <= ref.out_bound(o, o_abs, delta, q.dtype)).all()), (b, h)
            assert lse[b, h] == z or abs(float(lse[b, h]) - z) <= delta, (b, h)


FORMATS = [("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e4m3"), ("e2m1", "e2m1")]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_sizes_and_formats(d, formats, dtype):
    pr = Problem(1, [70, 1, 33], d=d, formats=formats, dtype=dtype).fill()
    check(pr, rows(pr, 4, dtype))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [1, 5, 40, 80, 100, 250])
def test_head_sizes_that_are_no_groups(d, dtype):
    pr = Problem(2, [50, 17], d=d, formats=("e2m1", "e4m3"), dtype=dtype, layout="inner").fill()
    check(pr, rows(pr, 6, dtype))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nkv,heads", [(1, 1), (1, 15), (1, 16), (2, 34), (1, 71), (5, 5), (1, 256)])
def test_groups_of_heads(nkv, heads, dtype):
    pr = Problem(3, [77, 20], nkv=nkv, d=64, dtype=dtype).fill()
    check(pr, rows(pr, heads, dtype))


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("group,d", [(17, 128), (24, 64), (32, 96), (33, 32), (71, 80)])
def test_wide_groups_over_enough_keys_for_two_tiles_of_heads(group, d, formats):
    # listed blocks, of which most are none: launches are cut by what may be listed, and the reference has few keys to look at
    held, block = [4200, 70, 0, 4095], 256
    pr = Problem(15, held, nkv=1, d=d, formats=formats, dtype=BF, block=block, most=8192).fill()
    q, listed = rows(pr, group, BF), 512 * 256 // (4 * -(-group // 32)) // block + 1
    lists = [[[i % 17 if i % 40 == 3 and held[b] else -1 for i in range(listed)]] for b in range(4)]
    check(pr, q, lists, cap=20.0, slopes=[0.01 * (h % 5) for h in range(group)])
    long = Problem(16, [3000], nkv=1, d=d, formats=formats, dtype=BF, most=132000, layout="pages", page=1024).fill()
    check(long, rows(long, group, BF))


@pytest.mark.parametrize("layout", ["slab", "pages", "inner"])
@pytest.mark.parametrize("held", [[0, 1, 2, 15], [16, 17, 31, 32], [33, 47, 48, 49], [127, 128, 129, 0], [300, 1, 255, 257]])
def test_lengths_and_layouts(held, layout):
    pr = Problem(4, held, d=96, layout=layout, page=16 if held[0] == 16 else 32).fill()
    check(pr, rows(pr, 4, BF))
    check(pr, rows(pr, 4, F32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("n", [1, 3])
def test_long_requests_in_parts(n, dtype):
    held = [5000, 1100, 3][:n]
    pr = Problem(5, held, nkv=1, d=128, formats=("e4m3", "e2m1"), dtype=dtype, layout="pages", page=64).fill()
    q = rows(pr, 4, dtype)
    assert hyp.mx_token_workspace_bytes(pr.cache, q.cuda()) > 0
    check(pr, q)
    check(pr, q, cap=20.0, slopes=[0.3, 0.01, 0.002, 0.0])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cap,scale", [(30.0, None), (0.5, 2.0), (5.0, 0.01), (50.0, 1.0)])
def test_capped_scores_and_slopes(cap, scale, dtype):
    pr = Problem(6, [200, 7, 64], d=64, dtype=dtype).fill()
    q = rows(pr, 4, dtype)
    check(pr, q, cap=cap, scale=scale)
    check(pr, q, cap=cap, scale=scale, slopes=[0.5, 0.1, 0.0, 0.02])
    check(pr, q, scale=scale, slopes=[0.5, 0.1, 0.0, 0.02])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("block,layout", [(16, "slab"), (32, "pages"), (64, "slab"), (16, "inner")])
def test_listed_blocks(block, layout, dtype):
    held = [20 * block - 5, 3 * block, 1, 0]
    pr = Problem(7, held, d=64, block=block, layout=layout, page=64, dtype=dtype).fill()
    q = rows(pr, 4, dtype)
    lists = [[[0, 3, 19, -1], [19, 18, 2, 5]], [[2, -1, -1, -1], [0, 1, 2, 3]], [[0, 1, 2, 3], [-1, -1, -1, -1]], [[0, 1, -1, 2], [-1, -1, -1, -1]]]
    check(pr, q, lists)
    check(pr, q, [[[x[1], -7, x[1], 1 << 30] for x in two] for two in lists])  # twice, and what is no block
    check(pr, q, [[[-1, -1, -1, x[0]] for x in two] for two in lists], slopes=[0.1, 0.2, 0.0, 0.3], cap=20.0)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_long_lists_in_parts(dtype):
    pr = Problem(8, [6000, 900], nkv=1, d=128, block=16, dtype=dtype, formats=("e2m1", "e2m1")).fill()
    q = rows(pr, 2, dtype)
    g = torch.Generator().manual_seed(1)
    lists = [[torch.randperm(375, generator=g)[:200].sort().values.tolist()], [list(range(57)) + [-1] * 143]]
    assert hyp.mx_token_workspace_bytes(pr.cache, q.cuda(), 200) > 0
    check(pr, q, lists)
    check(pr, q, [[[-1] * 199 + [3]], [[-1] * 200]])


def test_selected_blocks_as_they_are_used():
    # what a step of generation does: the new row is cached, blocks are chosen, and read
    pr = Problem(9, [700, 300, 64], d=128, block=32, dtype=BF, layout="pages", page=64, formats=("e4m3", "e2m1"))
    pr.write([0, 0, 0], [690, 290, 54])
    for turn in range(10):
        pr.write([690 + turn, 290 + turn, 54 + turn], [691 + turn, 291 + turn, 55 + turn], single=True)
    q = rows(pr, 8, BF)
    blocks = hyp.mx_select(pr.cache, q.cuda(), 6, sink=1, recent=2)
    k = pr.values()[0]
    want = []
    for b, held in enumerate(pr.held):
        for c in range(2):
            lo, hi = ref.bounds(k[b][:, c], 32)
            want.append(ref.select(q[b, 4 * c:4 * c + 4], lo, hi, held, 32, 6, 1, 2))
    assert blocks.cpu().reshape(6, 6).tolist() == want
    check(pr, q, blocks.tolist())
    every = hyp.mx_select(pr.cache, q.cuda(), 30)  # more than there are: all keys, in parts of another size
    check(pr, q, got=hyp.mx_token(pr.cache, hyp.AttnRule(128 ** -0.5), q.cuda(), blocks=every))


def test_strided_rows_and_results():
    pr = Problem(10, [60, 40], d=40, dtype=BF).fill()
    q = rows(pr, 4, BF)
    wide = torch.zeros((2, 7, 45), dtype=BF, device="cuda")
    wide[:, 1:5, 2:42] = q.cuda()
    out = torch.full((2, 9, 50), 7.0, dtype=BF, device="cuda")
    lse = torch.zeros((2, 4), device="cuda")
    got = hyp.mx_token(pr.cache, hyp.AttnRule(40 ** -0.5), wide[:, 1:5, 2:42], out=out[:, 2:6, 3:43], lse=lse)
    check(pr, q, got=(got[0], lse))
    out[:, 2:6, 3:43] = 7.0
    assert bool((out == 7.0).all())
    heads = q.cuda().transpose(0, 1).contiguous().transpose(0, 1)  # heads outside the rows
    check(pr, q, got=hyp.mx_token(pr.cache, hyp.AttnRule(40 ** -0.5), heads))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_keys_that_are_not_seen_have_no_influence_whatever_they_hold(dtype):
    # NaN in codes and scales behind the last key and in blocks that are not listed (Problem fills all of them with random bytes), and in key 0
    pr = Problem(11, [40, 100], d=64, block=16, dtype=dtype)
    pr.rows_k[1][0, :, 3], pr.rows_v[1][0, :, 5] = math.nan, math.inf
    pr.rows_v[0][20, :, 7] = math.nan
    pr.fill()
    q = rows(pr, 4, dtype)
    check(pr, q, [[[0, 2, -1], [2, 0, 0]], [[1, 2, 6], [-1, -1, 5]]])
    out, lse = hyp.mx_token(pr.cache, hyp.AttnRule(0.125), q.cuda(), blocks=torch.tensor([[[0], [1]], [[0], [1]]], dtype=torch.int32).cuda())
    nan = out.isnan().cpu()
    group = lambda b, h, g: bool(nan[b, h, 32 * g:32 * g + 32].all())  # noqa: E731
    assert not nan[0, :2].any() and group(0, 2, 0) and group(0, 3, 0) and not nan[0, 2:, 32:].any() and not lse[0].isnan().any()
    assert nan[1, :2].all() and not nan[1, 2:].any() and lse[1, :2].isnan().all()  # a key that is seen and NaN
    assert hyp.mx_token(pr.cache, hyp.AttnRule(0.125), q.cuda())[0][1].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_what_lies_behind_the_last_key_does_not_move_a_bit(dtype):
    # zeros, random bytes and the largest numbers there, which a cap would treat in its form for large scores
    got = []
    for behind in (0, None, 0x7e):
        pr = Problem(17, [37, 75, 5], d=64, formats=("e4m3", "e4m3"), dtype=dtype, block=0, most=96).fill()
        if behind is not None:
            for b, h in enumerate(pr.held):
                for t in (pr.k, pr.v):
                    t[b, :, h:] = behind
                for t in (pr.ks, pr.vs):
                    t[b, :, :, h:] = 200 if behind else 127
        q = torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(18)).to(dtype)
        for cap in (0.0, 40.0):
            rule = hyp.AttnRule(0.125, cap=cap, slopes=torch.tensor([0.3, 0.1, 0.01, 0.77]).cuda())
            got.append(hyp.mx_token(pr.cache, rule, q.cuda()))
    for out, lse in got[2:]:
        assert any(torch.equal(out, a) and torch.equal(lse, b) for a, b in got[:2])
    assert all(torch.equal(x, y) for i in (0, 1) for x, y in zip(got[i], got[i + 4]))


def test_rows_of_infinities_and_of_scores_beyond_floats():
    pr = Problem(12, [50], nkv=1, d=32, formats=("e4m3", "e4m3"), dtype=F32).fill()
    q = rows(pr, 3, F32)
    q[0, 1, 4], q[0, 2, 5] = math.nan, math.inf
    out, lse = hyp.mx_token(pr.cache, hyp.AttnRule(1.0), q.cuda())
    assert not out[0, 0].isnan().any() and out[0, 1:].isnan().all() and lse[0, 1:].isnan().all()
    check(pr, torch.zeros((1, 3, 32)))
    # large scores, one of which has all the weight; a large common part that the maximum takes away
    pr = Problem(13, [50], nkv=1, d=32, formats=("e4m3", "e4m3"), dtype=F32, spread=1e9).fill()
    check(pr, rows(pr, 3, F32) * 1e9, scale=1.0)


def test_equal_calls_have_equal_bits():
    pr = Problem(14, [3000, 2100], nkv=2, d=128, dtype=BF).fill()
    q = rows(pr, 8, BF).cuda()
    a = [hyp.mx_token(pr.cache, hyp.AttnRule(0.1), q) for _ in range(4)]
    assert all(torch.equal(a[0][0], x[0]) and torch.equal(a[0][1], x[1]) for x in a)


def test_problems_drawn_at_random():
    g = torch.Generator().manual_seed(77)
    draw = lambda *x: x[int(torch.randint(0, len(x), (1,), generator=g))]  # noqa: E731
    for case in range(40):
        nkv, group, d, dtype = draw(1, 2, 3), draw(1, 2, 4, 7, 17), draw(16, 48, 64, 80, 128, 144), draw(F32, BF)
        held = [draw(0, 1, 16, 30, 65, 128, 190, 260) for _ in range(draw(1, 2, 4))]
        block, layout = draw(16, 32), draw("slab", "pages", "inner")
        pr = Problem(100 + case, held, nkv=nkv, d=d, formats=draw(*FORMATS), block=block, layout=layout, page=draw(32, 64, 128), dtype=dtype, most=max(held) + draw(0, 1, 40) or 1).fill()
        heads = nkv * group
        lists = None
        if draw(0, 1):
            listed = draw(1, 3, 9)
            lists = [[[draw(-1, *range(max(1, -(-h // block) + 1))) for _ in range(listed)] for _ in range(nkv)] for h in held]
        check(pr, rows(pr, heads, dtype), lists, cap=draw(0.0, 0.0, 15.0), slopes=draw(None, [0.05 * (h % 5) for h in range(heads)]))
