"""mx_write and mx_read against the formats' definition: every code, scale and bound, layouts, parts of rows, rows and slots that nothing names."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import mx_reference as ref
from tests.mx_problem import BF, F32, Problem

pytestmark = pytest.mark.gpu

nan_as = lambda t: t.double().cpu().nan_to_num(nan=7e77, posinf=8e77, neginf=-8e77)  # noqa: E731


def check(pr):
    """The cache's codes and bounds are those of the rows"""
    k, v = pr.values()
    for b, held in enumerate(pr.held):
        for c in range(pr.nkv):
            for j in range(held):
                got = pr.codes(b, c, j)
                assert torch.equal(nan_as(got[0]), nan_as(k[b][j, c])) and torch.equal(nan_as(got[1]), nan_as(v[b][j, c])), (b, c, j)
            if pr.block and held:
                lo, hi = ref.bounds(k[b][:held, c], pr.block)
                for i in range(lo.shape[0]):
                    page, at = pr.place(b, i, pr.lo.shape[2])
                    assert torch.equal(nan_as(pr.lo[page, c, at]), nan_as(lo[i])) and torch.equal(nan_as(pr.hi[page, c, at]), nan_as(hi[i])), (b, c, i)


def check_read(pr, dtype=F32, first=None, keys=None, layout="heads"):
    k, v = pr.values()
    n, room = len(pr.held), pr.most if keys is None else keys
    shape = (n, pr.nkv, room, pr.d)
    out = [torch.full(shape, 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    if layout == "keys":
        out = [torch.full((n, room, pr.nkv, pr.d + 1), 5.0, dtype=dtype, device="cuda")[..., :pr.d].transpose(1, 2) for _ in range(2)]
    hyp.mx_read(pr.cache, *out, first=None if first is None else torch.tensor(first, dtype=torch.int32).cuda())
    for x, want in zip(out, (k, v)):
        for b, held in enumerate(pr.held):
            a = 0 if first is None else min(max(first[b], 0), held)
            count = min(held - a, room)
            assert torch.equal(nan_as(x[b, :, :count]), nan_as(want[b][a:a + count].transpose(0, 1).to(dtype)))
            assert bool((x[b, :, count:] == 5.0).all())


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e4m3"), ("e2m1", "e2m1")])
def test_rows_become_the_numbers_of_the_formats(dtype, formats):
    pr = Problem(1, [37, 1, 64, 0, 16], d=64, formats=formats, dtype=dtype).fill()
    check(pr)
    check_read(pr, dtype)
    check_read(pr, BF if dtype == F32 else F32)


@pytest.mark.parametrize("layout", ["slab", "pages", "inner"])
@pytest.mark.parametrize("d", [1, 7, 32, 33, 80, 96, 128, 160, 200, 256])
def test_head_sizes_and_layouts(d, layout):
    pr = Problem(2, [19, 40], nkv=3, d=d, formats=("e2m1", "e4m3"), layout=layout, dtype=BF if d % 2 else F32).fill()
    check(pr)
    check_read(pr, layout="keys")


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_ties_subnormals_and_the_ends_of_the_range(fmt):
    # every midpoint of two numbers and its neighbours, at scales up to the ends of a float; groups of nothing, of infinities and NaN
    f, pr = ref.FORMATS[fmt], Problem(3, [48], nkv=2, d=64, formats=(fmt, fmt))
    table = [ref.number(fmt, c) for c in range(127 if fmt == "e4m3" else 8)]
    mids = [(a + b) / 2 for a, b in zip(table, table[1:])]
    values = [w for m in mids for w in (m, math.nextafter(m, 0), math.nextafter(m, 1e9))] + table
    x = torch.tensor(values, dtype=torch.float64)
    rows = torch.zeros((48, 2, 64), dtype=torch.float32)
    for j in range(48):
        for c in range(2):
            at = (j * 2 + c) * 60 % len(values)
            part = torch.cat([x] * 5)[at:at + 62]
            s = 2.0 ** [0, 5, -20, 60, -60, f["high"] - 1, -117, -126][j % 8]
            rows[j, c, :62] = (part * s * torch.where(torch.arange(62) % 3 == 0, -1.0, 1.0)).float()
            rows[j, c, 62] = rows[j, c, 0 if j % 2 else 33] = f["most"] * s  # one group, or both, go by the largest number
    rows[5, 0, 3], rows[5, 1, 40], rows[6, 0] = math.inf, math.nan, 0.0
    rows[7, 1] = 3.4e38
    rows[8, 0] = torch.full((64,), -1e-42)
    pr.rows_k, pr.rows_v = [rows], [rows.flip(0)]
    pr.fill()
    check(pr)
    check_read(pr)


@pytest.mark.parametrize("layout", ["slab", "pages", "inner"])
@pytest.mark.parametrize("block", [0, 16, 32])
def test_caches_grow_by_prompts_and_by_single_rows(block, layout):
    held = [70, 33, 5, 48]
    pr = Problem(4, held, d=96, block=block, layout=layout)
    pr.write([0] * 4, [17, 16, 0, 31])
    pr.write([17, 16, 0, 31], [18, 33, 0, 47])
    pr.write([18, 33, 0, 47], [63, 33, 1, 47])
    pr.held, want = [63, 33, 1, 47], held
    check(pr)
    pr.held = want
    for turn in range(7):  # rows of requests that are done go where they were
        pr.write([min(63 + turn, 69), 32, min(1 + turn, 4), 47], [min(64 + turn, 70), 33, min(2 + turn, 5), 48], single=True)
    check(pr)
    check_read(pr)


def test_bounds_of_keys_that_are_written_again_hold_both():
    pr = Problem(5, [40], nkv=1, d=32, formats=("e4m3", "e4m3")).fill()
    old = pr.values()[0][0]
    pr.rows_k[0] = pr.rows_k[0].clone()
    pr.rows_k[0][20:30] = torch.randn((10, 1, 32), generator=pr.gen)
    pr.write([20], [30])
    new = pr.values()[0][0]
    lo, hi = pr.lo[0, 0, 1].double().cpu(), pr.hi[0, 0, 1].double().cpu()
    both = torch.cat([old[16:32, 0], new[20:30, 0]])
    assert torch.equal(lo, both.amin(0)) and torch.equal(hi, both.amax(0))
    pr.write([16], [40])  # from the block's first key on they begin again
    lo, hi = ref.bounds(new[:, 0], 16)
    assert torch.equal(pr.lo[0, 0, :3].double().cpu(), lo) and torch.equal(pr.hi[0, 0, :3].double().cpu(), hi)


@pytest.mark.parametrize("d", [64, 40, 33])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_stored_numbers_come_back_as_rows(dtype, d):
    pr = Problem(6, [21, 9], d=d, dtype=dtype)
    out = [torch.full((30, 2, d + 5), 3.0, dtype=dtype, device="cuda") for _ in range(2)]
    pr.write([0, 0], [21, 9], k_out=out[0][..., :d], v_out=out[1][..., :d])
    k, v = pr.write([0, 0], [21, 9], k_out=None, v_out=None)
    for x, want, rest in zip(out, pr.values(), out):
        assert torch.equal(x[..., :d].double().cpu(), torch.cat(want).to(dtype).double()) and bool((rest[..., d:] == 3.0).all())
    # in place
    start = torch.tensor([0, 21, 30], dtype=torch.int32).cuda()
    hyp.mx_write(pr.cache, k, v, q_start=start, k_out=k, v_out=v)
    assert torch.equal(k, out[0][..., :d]) and torch.equal(v, out[1][..., :d])
    check(pr)


def test_rows_that_no_key_is_for_and_keys_that_no_row_is_for_stay():
    # more rows than keys: the newest count; wrong lengths and ranges are cut; rows behind the last sequence stay
    pr = Problem(7, [10, 20], nkv=1, d=32, formats=("e4m3", "e4m3"), block=16, most=24)
    codes, scales = pr.k.clone(), pr.ks.clone()
    k = torch.randn((40, 1, 32), generator=pr.gen).cuda()
    out = [torch.full_like(k, 9.0) for _ in range(2)]
    pr.lens.copy_(torch.tensor([4, 100], dtype=torch.int32))
    start = torch.tensor([3, 9, 33], dtype=torch.int32).cuda()
    hyp.mx_write(pr.cache, k, k, q_start=start, k_out=out[0], v_out=out[1])
    want = ref.stored_rows("e4m3", k[:, 0].cpu())
    assert bool((out[0][:5] == 9.0).all()) and bool((out[0][33:] == 9.0).all())       # rows 3 and 4 are for keys -2 and -1
    assert torch.equal(out[0][5:33, 0].double().cpu(), want[5:33])
    pr.held, pr.rows_k = [4, 24], [k[5:9].cpu(), k[9:33].cpu()]
    pr.rows_v = pr.rows_k
    check(pr)
    assert torch.equal(pr.k[0, 0, 4:], codes[0, 0, 4:]) and torch.equal(pr.ks[0, 0, :, 4:], scales[0, 0, :, 4:]) and torch.equal(pr.k[1, 0, 24:], codes[1, 0, 24:])
    # ranges that are no ranges: nothing outside the tensors
    for bad in ([5, 2, 90], [-7, 50, 60], [2 ** 31 - 1, -2 ** 31, 7]):
        hyp.mx_write(pr.cache, k, k, q_start=torch.tensor(bad, dtype=torch.int32).cuda())
    pr.lens.copy_(torch.tensor([-5, -2 ** 31], dtype=torch.int32))
    codes = pr.k.clone()
    hyp.mx_write(pr.cache, k, k, q_start=start)
    torch.cuda.synchronize()
    assert torch.equal(pr.k, codes)


def test_pages_outside_the_pool_are_cut():
    pr = Problem(8, [64, 64], nkv=1, d=32, block=16, layout="pages").fill()
    table = pr.cache.page_table
    table.copy_(torch.tensor([[-1, 2 ** 31 - 1], [-2 ** 31, 1 << 20]], dtype=torch.int32))
    pr.write([0, 0], [64, 64])
    out = [torch.zeros((2, 1, 64, 32), device="cuda") for _ in range(2)]
    hyp.mx_read(pr.cache, *out)
    hyp.mx_token(pr.cache, hyp.AttnRule(1.0), torch.randn((2, 2, 32), generator=pr.gen).cuda())
    hyp.mx_select(pr.cache, torch.randn((2, 2, 32), generator=pr.gen).cuda(), 2)
    torch.cuda.synchronize()


@pytest.mark.parametrize("first,keys", [([5, 0, 12], None), ([0, 0, 0], 9), ([30, 3, 40], 4), ([-5, 2 ** 31 - 1, -2 ** 31], 12)])
@pytest.mark.parametrize("layout", ["slab", "pages"])
def test_reading_from_a_key_on(first, keys, layout):
    pr = Problem(9, [37, 16, 40], d=128, formats=("e4m3", "e2m1"), layout=layout).fill()
    check_read(pr, BF, first, keys)


def test_offsets_beyond_32_bits():
    # a slab of more than 2^31 bytes: the last request's keys lie behind them
    room, n, d = 1 << 20, 36, 64
    k = torch.zeros((n, 1, room, 64), dtype=torch.uint8, device="cuda")
    ks = torch.zeros((n, 1, 2, room), dtype=torch.uint8, device="cuda")
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    lens[-1] = room
    v, vs = torch.zeros_like(k), torch.zeros_like(ks)
    cache = hyp.MxCache(k, v, ks, vs, lens, d, block_keys=64)
    x = torch.randn((50, 1, d), generator=torch.Generator().manual_seed(10))
    start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    start[-1] = 50
    hyp.mx_write(cache, x.cuda(), x.cuda(), q_start=start)
    want = ref.stored_rows("e4m3", x[:, 0])
    first = torch.full((n,), room - 50, dtype=torch.int32, device="cuda")
    out = [torch.zeros((n, 1, 50, d), device="cuda") for _ in range(2)]
    hyp.mx_read(cache, *out, first=first)
    assert torch.equal(out[0][-1, 0].double().cpu(), want) and torch.equal(out[1][-1, 0].double().cpu(), want)
    blocks = torch.full((n, 1, 1), room // 64 - 1, dtype=torch.int32, device="cuda")
    q = torch.ones((n, 1, d), device="cuda")
    got, lse = hyp.mx_token(cache, hyp.AttnRule(0.125), q, blocks=blocks)
    keys = torch.cat([torch.zeros((14, d), dtype=torch.float64), want])  # the block's other keys are zeros
    o, z, o_abs, delta = ref.attend(q[-1, 0].cpu(), keys, keys, list(range(64)), scale=0.125)
    assert bool(((got[-1, 0].double().cpu() - o).abs() <= ref.out_bound(o, o_abs, delta, F32)).all()) and abs(float(lse[-1, 0]) - z) <= delta
    assert bool((got[:-1] == 0).all()) and bool((lse[:-1] == -math.inf).all())


@pytest.mark.parametrize("n", [511, 512, 513, 1100])
def test_many_requests(n):
    # starts and lengths of up to 512 requests are read at once, of more request by request
    held = [(i * 7) % 5 for i in range(n)]
    pr = Problem(11, held, nkv=1, d=32, formats=("e4m3", "e4m3"), block=16, layout="pages", page=16).fill()
    room = torch.zeros((n, 1, 4, 32), device="cuda")
    out = [room, torch.zeros_like(room)]
    hyp.mx_read(pr.cache, *out)
    want = torch.cat(pr.values()[0])[:, 0]
    got = torch.cat([out[0][b, 0, :h] for b, h in enumerate(held)])
    assert torch.equal(got.double().cpu(), want)


def test_keys_far_apart():
    # a key stride just below what is allowed, in a block of 512 keys: bytes beyond 32 bits from the block's first key
    stride, keys, d, room = (1 << 24) - 16, 300, 32, 512
    k = torch.empty(stride * room, dtype=torch.uint8, device="cuda").view(1, 1, room, stride)[..., :32]
    small = lambda: torch.zeros((1, 1, room, 32), dtype=torch.uint8, device="cuda")  # noqa: E731
    scale = lambda: torch.zeros((1, 1, 1, room), dtype=torch.uint8, device="cuda")  # noqa: E731
    lens = torch.tensor([keys], dtype=torch.int32, device="cuda")
    lo, hi = (torch.zeros((1, 1, 1, d), dtype=BF, device="cuda") for _ in range(2))
    cache = hyp.MxCache(k, small(), scale(), scale(), lens, d, most=keys, lo=lo, hi=hi)
    x = torch.randn((keys, 1, d), generator=torch.Generator().manual_seed(12))
    start = torch.tensor([0, keys], dtype=torch.int32, device="cuda")
    hyp.mx_write(cache, x.cuda(), x.cuda(), q_start=start)
    out = [torch.zeros((1, 1, keys, d), device="cuda") for _ in range(2)]
    hyp.mx_read(cache, *out)
    want = ref.stored_rows("e4m3", x[:, 0])
    assert torch.equal(out[0][0, 0].double().cpu(), want) and torch.equal(out[1][0, 0].double().cpu(), want)
    assert torch.equal(lo[0, 0, 0].double().cpu(), want.amin(0))
