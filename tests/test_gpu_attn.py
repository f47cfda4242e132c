"""Attention over a shared prefix and own keys (hyp_attn.h) against its formulas in 64 bits: types, head layouts, lengths, strides,
pages, masks that leave rows empty, numbers in places that no row sees, streams, graphs."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import attn_reference as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAN, INF = math.nan, math.inf


class Problem:
    """A cache, rows and a rule, drawn on the host; the same values on the device in the layout asked for."""

    def __init__(self, seed, dtype, nq, nkv, d, held, rows=None, prefix=0, cap=0.0, slopes=False, docs=None, see_all=None, page=0, layout="heads",
                 room=None, pos=False, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        n, self.most = len(held), max(held + [1])
        room = room or self.most + 3
        self.dtype, self.nq, self.nkv, self.d, self.held, self.prefix_len = dtype, nq, nkv, d, held, prefix
        self.token = rows is None
        self.rows = [1] * n if self.token else rows
        total = sum(self.rows)
        rnd = lambda *s: (torch.randn(s, generator=g) * sigma).to(dtype)  # noqa: E731
        self.k, self.v = rnd(n, nkv, room, d), rnd(n, nkv, room, d)
        for b, h in enumerate(held):  # what no request holds must not matter
            self.k[b, :, h:], self.v[b, :, h:] = NAN, NAN
        self.q = rnd(total, nq, d)
        self.pk, self.pv = (rnd(nkv, prefix, d), rnd(nkv, prefix, d)) if prefix else (None, None)
        self.scale, self.cap = 1.0 / math.sqrt(d), cap
        self.slopes = torch.tensor([2.0 ** (-1 - h % 7) / 4 for h in range(nq)]) if slopes else None
        self.see_all = see_all
        self.q_doc = self.key_doc = None
        if docs:
            self.key_doc = torch.randint(-1, docs, (n, nkv, room), generator=g, dtype=torch.int32).sort(-1).values
            self.q_doc = torch.randint(-1, docs + 2, (total,), generator=g, dtype=torch.int32)  # some ids that no key has
        self.key_pos = self.q_pos = None
        if pos:
            self.key_pos = torch.randint(0, 500, (n, nkv, room), generator=g, dtype=torch.int32)
            self.q_pos = torch.randint(0, 900, (total,), generator=g, dtype=torch.int32)
        self.page, self.layout, self.room, self.g = page, layout, room, g

    def device(self):
        c = lambda t: None if t is None else t.cuda()  # noqa: E731
        n = len(self.held)

        def tensor(x):
            if self.layout == "tokens":  # [n, key, head, d]
                return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            if self.layout == "odd":     # every row starts 1 element off
                big = torch.full(x.shape[:3] + (x.shape[3] + 3,), NAN, dtype=x.dtype)
                big[..., 1:1 + x.shape[3]] = x
                return big.cuda()[..., 1:1 + x.shape[3]]
            return x.cuda()
        table = None
        k, v = self.k, self.v
        if self.page:
            pages = -(-self.room // self.page)
            table = torch.randperm(n * pages, generator=self.g).reshape(n, pages).to(torch.int32)
            pools = []
            for x in (k, v):
                full = torch.full((n, self.nkv, pages * self.page, self.d), NAN, dtype=x.dtype)
                full[:, :, :self.room] = x
                pool = torch.full((n * pages, self.nkv, self.page, self.d), NAN, dtype=x.dtype)
                pool[table.reshape(-1).long()] = full.reshape(n, self.nkv, pages, self.page, self.d).permute(0, 2, 1, 3, 4).reshape(-1, self.nkv, self.page, self.d)
                pools.append(pool)
            k, v = pools
        lens = torch.tensor(self.held, dtype=torch.int32).cuda()
        self.cache = hyp.AttnCache(tensor(k), tensor(v), lens, page_table=c(table), most=self.most, prefix_k=None if self.pk is None else tensor(self.pk[None])[0],
                                   prefix_v=None if self.pv is None else tensor(self.pv[None])[0], key_pos=c(self.key_pos), key_doc=c(self.key_doc))
        self.rule = hyp.AttnRule(self.scale, cap=self.cap, slopes=c(self.slopes))
        qd = tensor(self.q[None])[0] if self.layout != "tokens" else self.q.cuda()
        start = torch.tensor([sum(self.rows[:i]) for i in range(n + 1)], dtype=torch.int32).cuda()
        return qd, start, c(self.q_pos), c(self.q_doc), None if self.see_all is None else torch.tensor(self.see_all, dtype=torch.int32).cuda()

    def reference(self, last=0):
        """out, lse, totals [n, nkv, most] and their bounds"""
        n, G = len(self.held), self.nq // self.nkv
        out, bound = (torch.zeros(self.q.shape, dtype=torch.float64) for _ in range(2))
        lse, lse_b = (torch.zeros(self.q.shape[:2], dtype=torch.float64) for _ in range(2))
        tot, tot_b = (torch.zeros((n, self.nkv, self.most), dtype=torch.float64) for _ in range(2))
        first = 0
        for b, (h, r) in enumerate(zip(self.held, self.rows)):
            sl = slice(first, first + r)
            for x in range(self.nq):
                c = x // G
                o, z, p, oa, de = ref.attend(
                    self.q[sl, x], self.k[b, c, :h], self.v[b, c, :h], [h - r + i for i in range(r)], scale=self.scale,
                    prefix=(self.pk[c], self.pv[c]) if self.prefix_len else None, cap=self.cap, slope=0.0 if self.slopes is None else float(self.slopes[x]),
                    see_all=0 if self.see_all is None or self.token else self.see_all[b], q_doc=None if self.q_doc is None else self.q_doc[sl].tolist(),
                    key_doc=None if self.key_doc is None else self.key_doc[b, c].tolist(), q_pos=None if self.q_pos is None else self.q_pos[sl].tolist(),
                    key_pos=None if self.key_pos is None else self.key_pos[b, c].tolist())
                out[sl, x], lse[sl, x] = o, z
                bound[sl, x] = ref.out_bound(o, oa, de, self.dtype)
                lse_b[sl, x] = de + 2.0 ** -21 * (1 + torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z)))
                lo = max(0, r - last) if last else 0
                tot[b, c, :h] += p[lo:].sum(0)
                tot_b[b, c, :h] += (p[lo:] * (3 * de[lo:, None] + 2.0 ** -19)).sum(0)
            first += r
        return out, lse, tot, bound, lse_b, tot_b + 1e-12


def close(got, want, bound, what):
    got = got.detach().double().cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    assert torch.equal(got[~torch.isfinite(want)], want[~torch.isfinite(want)]), what
    ok = torch.isfinite(want)
    worst = ((got - want).abs() / bound)[ok]
    assert worst.numel() == 0 or float(worst.max()) <= 1.0, f"{what}: {float(worst.max())} of the bound"


def check_prompt(pr, last=0, received=True):
    q, start, q_pos, q_doc, see = pr.device()
    out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start, see_all=see, q_pos=q_pos, q_doc=q_doc)
    w_out, w_lse, w_tot, b_out, b_lse, b_tot = pr.reference(last)
    close(lse, w_lse, b_lse, "lse")
    close(out, w_out, b_out, "out")
    if received:
        base = torch.rand((len(pr.held), pr.nkv, pr.most + 2), generator=pr.g).cuda()
        got = torch.full_like(base, -7.0)
        hyp.attn_received(pr.cache, pr.rule, q, start, lse, base, last=last, see_all=see, q_pos=q_pos, q_doc=q_doc, totals_out=got)
        close(got[..., :pr.most], base[..., :pr.most].double().cpu() + w_tot, b_tot + 2.0 ** -23 * (1 + w_tot), "totals")
        assert bool((got[..., pr.most:] == -7.0).all())
        hyp.attn_received(pr.cache, pr.rule, q, start, lse, base, last=last, see_all=see, q_pos=q_pos, q_doc=q_doc)  # in place
        assert torch.equal(base[..., :pr.most], got[..., :pr.most])
    return out


def check_token(pr, totals=True):
    q, _, q_pos, q_doc, _ = pr.device()
    base = torch.rand((len(pr.held), pr.nkv, pr.most), generator=pr.g).cuda() if totals else None
    got = torch.empty_like(base) if totals else None
    out, lse = hyp.attn_token(pr.cache, pr.rule, q, q_pos=q_pos, q_doc=q_doc, totals=base, totals_out=got)
    w_out, w_lse, w_tot, b_out, b_lse, b_tot = pr.reference()
    close(lse, w_lse, b_lse, "lse")
    close(out, w_out, b_out, "out")
    if totals:
        close(got, base.double().cpu() + w_tot, b_tot + 2.0 ** -23 * (1 + w_tot), "totals")
        hyp.attn_token(pr.cache, pr.rule, q, q_pos=q_pos, q_doc=q_doc, totals=base)
        assert torch.equal(base, got)
    return out


HEADS = [(4, 2, 64), (8, 2, 128), (5, 1, 80), (3, 3, 96), (7, 1, 40), (2, 1, 256), (3, 1, 33), (6, 2, 200)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nq,nkv,d", HEADS)
def test_prompt_head_layouts(dtype, nq, nkv, d):
    check_prompt(Problem(d, dtype, nq, nkv, d, held=[37, 1, 70, 140], rows=[37, 1, 5, 66], prefix=19), last=9)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nq,nkv,d", HEADS)
def test_token_head_layouts(dtype, nq, nkv, d):
    check_token(Problem(d + 1, dtype, nq, nkv, d, held=[37, 1, 0, 140, 259], prefix=75))


@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
def test_prompt_lengths_around_the_tiles(n):
    check_prompt(Problem(n, BF, 2, 1, 64, held=[n, 2 * n], rows=[n, n]))


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 1025])
@pytest.mark.parametrize("prefix", [0, 1, 129])
def test_token_lengths_around_the_tiles(n, prefix):
    check_token(Problem(n, BF, 4, 2, 128, held=[n, max(n - 1, 0)], prefix=prefix))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rule", [dict(cap=5.0), dict(cap=50.0, sigma=4.0), dict(slopes=True), dict(cap=2.0, slopes=True, pos=True), dict(docs=3),
                                  dict(docs=4, see_all=[0, 300, 17]), dict(see_all=[1, 64, 80]), dict(docs=2, slopes=True, pos=True, cap=30.0)])
def test_rules_and_masks(dtype, rule):
    pr = Problem(11, dtype, 4, 2, 128, held=[90, 33, 150], rows=[90, 20, 77], prefix=0 if "docs" in rule else 40, **rule)
    check_prompt(pr, last=30)
    tok = Problem(12, dtype, 4, 2, 128, held=[90, 33, 400], prefix=0 if "docs" in rule else 40, **{k: v for k, v in rule.items() if k != "see_all"})
    check_token(tok)


@pytest.mark.parametrize("page", [1, 16, 32, 64, 128])
@pytest.mark.parametrize("layout", ["heads", "tokens", "odd"])
def test_pages_and_strides(page, layout):
    check_prompt(Problem(page, BF, 4, 2, 64, held=[100, 40, 213], rows=[60, 40, 130], prefix=70, page=page, layout=layout, docs=3))
    check_token(Problem(page, BF, 4, 2, 64, held=[100, 40, 333], prefix=70, page=page, layout=layout))
    check_token(Problem(page, F32, 4, 2, 64, held=[100, 40, 333], prefix=70, page=page, layout=layout))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_requests_without_rows_or_keys(dtype):
    check_prompt(Problem(3, dtype, 4, 2, 64, held=[0, 50, 7, 1], rows=[0, 0, 7, 1]))
    # more rows than keys: the first rows have a negative index and see the shared keys only
    pr = Problem(4, dtype, 4, 2, 64, held=[3, 10], rows=[8, 10], prefix=5)
    check_prompt(pr)
    check_prompt(Problem(4, dtype, 4, 2, 64, held=[3, 10], rows=[8, 10]))  # ... or nothing at all
    check_token(Problem(5, dtype, 4, 2, 64, held=[0, 0, 1]))


def test_no_rows_at_all():
    pr = Problem(3, BF, 4, 2, 64, held=[5, 5], rows=[0, 0])
    q, start, *_ = pr.device()
    out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    totals = torch.rand((2, 2, 5)).cuda()
    got = hyp.attn_received(pr.cache, pr.rule, q, start, lse, totals, totals_out=torch.empty_like(totals))
    assert torch.equal(got, totals)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("held,prefix", [([1500], 0), ([700, 40], 900), ([2], 2100)])
def test_few_rows_over_many_keys_are_cut(dtype, held, prefix):
    check_prompt(Problem(6, dtype, 4, 2, 64, held=held, rows=[min(2, h) for h in held], prefix=prefix, cap=20.0))


@pytest.mark.parametrize("n", [1, 8, 9, 33])
def test_batches_behind_one_prefix(n):
    # up to 32 pairs a KV head the waves share the keys, beyond each has rows of its own
    check_token(Problem(n, BF, 8, 2, 128, held=[(37 * b) % 90 for b in range(n)], prefix=333))
    check_token(Problem(n, F32, 8, 2, 128, held=[(37 * b) % 90 for b in range(n)], prefix=333), totals=False)


def test_more_than_32_heads_a_group():
    check_token(Problem(1, BF, 80, 2, 64, held=[100, 7], prefix=50))
    check_prompt(Problem(1, BF, 80, 2, 64, held=[20, 7], rows=[20, 3], prefix=50))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_numbers_that_a_row_does_not_see(dtype, bad):
    for d in (64, 33):
        pr = Problem(8, dtype, 4, 2, d, held=[80, 50], rows=[80, 30], docs=3, prefix=10)
        pr.key_doc[:] = torch.arange(pr.key_doc.shape[2], dtype=torch.int32) // 27
        pr.q_doc[:] = torch.tensor([(i // 27) for i in range(80)] + [(i + 20) // 27 for i in range(30)], dtype=torch.int32)
        check_prompt(pr)
        pr.k[:, :, 30] = bad      # an id 1 key: rows of the other ids, and earlier rows, go on as before
        pr.v[:, :, 30] = bad
        q, start, _, q_doc, _ = pr.device()
        out, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start, q_doc=q_doc)
        own = torch.tensor([i for i in range(80)] + [i + 20 for i in range(30)])
        away = (pr.q_doc != 1) | (own < 30)
        assert torch.isfinite(out[away.cuda()]).all() and torch.isfinite(lse[away.cuda()]).all()
        w_out, w_lse, _, b_out, b_lse, _ = pr.reference()
        close(out[away.cuda()], w_out[away], b_out[away], "rows that do not see it")
        close(lse[away.cuda()], w_lse[away], b_lse[away], "their lse")
        if bad != bad:
            assert torch.isnan(out[~away.cuda()]).all()
    tok = Problem(9, dtype, 4, 2, 64, held=[80, 50], docs=3)
    tok.key_doc[:] = torch.arange(tok.key_doc.shape[2], dtype=torch.int32) // 27
    tok.q_doc[:] = 1
    tok.k[:, :, 3], tok.v[:, :, 3] = bad, bad
    check_token(tok)


def test_sums_that_leave_the_range_on_the_way():
    # probabilities may be up to 2^8 above their last maximum: values near the end of the range then pass it, the result does not
    pr = Problem(10, F32, 2, 1, 64, held=[64], rows=[64])
    pr.v[:] = 3e38
    pr.k[:], pr.q[:] = 0.0, 0.0
    pr.k[:, :, :, 0], pr.q[:, :, 0] = torch.arange(pr.k.shape[2]) * 0.08, 8.0
    q, start, *_ = pr.device()
    out, _ = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    assert torch.isfinite(out).all() and float((out / 3e38 - 1).abs().max()) < 1e-5


def test_offsets_beyond_31_bits():
    n, nkv, room, d = 3, 8, 700_000, 128  # 2.15e9 values in a slab
    held = [5, 3, 600]
    k, v = (torch.empty((n, nkv, room, d), dtype=BF, device="cuda") for _ in range(2))
    pr = Problem(2, BF, 8, 8, d, held=held, prefix=20)
    pr.device()
    lens = torch.tensor(held, dtype=torch.int32, device="cuda")
    k[:, :, :600], v[:, :, :600] = pr.k[:, :, :600].cuda(), pr.v[:, :, :600].cuda()
    cache = hyp.AttnCache(k, v, lens, most=600, prefix_k=pr.pk.cuda(), prefix_v=pr.pv.cuda())
    out, lse = hyp.attn_token(cache, pr.rule, pr.q.cuda())
    w_out, w_lse, _, b_out, b_lse, _ = pr.reference()
    close(out, w_out, b_out, "out")
    close(lse, w_lse, b_lse, "lse")
    # the last keys of a request: one long page table entry past 2^31 elements
    count = n * nkv * room // 1024
    pool_k, pool_v = (x.view(-1)[:count * 1024 * d].view(count, 8, 128, d) for x in (k, v))
    pages = torch.tensor([[16404 - b] * 5 for b in range(n)], dtype=torch.int32, device="cuda") - torch.arange(5, dtype=torch.int32, device="cuda") * 3
    assert int(pages.max()) < pool_k.shape[0] and len(set(pages.flatten().tolist())) == 15
    for b in range(n):
        for i in range(5):
            part = slice(i * 128, min((i + 1) * 128, 600))
            pool_k[pages[b, i], :, :part.stop - part.start] = pr.k[b, :, part].cuda()
            pool_v[pages[b, i], :, :part.stop - part.start] = pr.v[b, :, part].cuda()
    cache = hyp.AttnCache(pool_k, pool_v, lens, page_table=pages, most=600, prefix_k=pr.pk.cuda(), prefix_v=pr.pv.cuda())
    out, lse = hyp.attn_token(cache, pr.rule, pr.q.cuda())
    close(out, w_out, b_out, "out")


def test_lengths_and_tables_on_the_device_are_cut_to_what_there_is():
    pr = Problem(2, BF, 4, 2, 64, held=[50, 50], page=16, prefix=10)
    q, *_ = pr.device()
    cache = pr.cache
    cache._keep[2].fill_(1 << 30)     # lens far beyond most: counts as most
    cache._keep[3][1] = -5            # pages outside the pool
    cache._keep[3][0, 2] = 1 << 29
    hyp.attn_token(cache, pr.rule, q, totals=torch.zeros((2, 2, 50), device="cuda"))
    cache._keep[2].fill_(-3)          # counts as none: the shared keys alone
    _, lse = hyp.attn_token(cache, pr.rule, q)
    assert torch.isfinite(lse).all()
    start = torch.tensor([0, 1 << 30, -7], dtype=torch.int32, device="cuda")
    hyp.attn_prompt(cache, pr.rule, q, start)
    torch.cuda.synchronize()


def test_outputs_of_the_callers_own():
    pr = Problem(21, BF, 4, 2, 64, held=[70, 9], rows=[70, 5], prefix=30)
    q, start, *_ = pr.device()
    want, lse = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    wide = torch.full((75, 4, 67), 9.0, dtype=BF, device="cuda")  # rows that cannot be stored four features at once
    out, lse2 = hyp.attn_prompt(pr.cache, pr.rule, q, start, out=wide[..., 1:65], lse=torch.empty_like(lse))
    assert torch.equal(out, want) and torch.equal(lse, lse2) and bool((wide[..., 0] == 9).all()) and bool((wide[..., 65:] == 9).all())
    tok = Problem(22, BF, 4, 2, 64, held=[70, 9], prefix=30)
    q, *_ = tok.device()
    want, _ = hyp.attn_token(tok.cache, tok.rule, q)
    ws = torch.empty(hyp.attn_workspace_bytes(tok.cache, tok.rule, q) + 16, dtype=torch.uint8, device="cuda")
    out, _ = hyp.attn_token(tok.cache, tok.rule, q, out=torch.empty((2, 8, 64), dtype=BF, device="cuda")[:, ::2], workspace=ws)
    assert torch.equal(out, want)


def test_other_streams_and_graphs():
    pr = Problem(23, BF, 8, 2, 128, held=[300, 41, 7], prefix=200, cap=30.0)
    q, *_ = pr.device()
    totals = torch.rand((3, 2, 300), device="cuda")
    into = torch.empty_like(totals)
    want, lse = hyp.attn_token(pr.cache, pr.rule, q, totals=totals, totals_out=into)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, lse2 = hyp.attn_token(pr.cache, pr.rule, q, totals=totals, totals_out=torch.empty_like(totals), stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    out, z, into2 = torch.empty_like(want), torch.empty_like(lse), torch.empty_like(totals)
    kept = torch.empty((3, 2, 20), dtype=torch.int32, device="cuda")
    small = hyp.AttnCache(*(torch.zeros((3, 2, 20, 128), dtype=BF, device="cuda") for _ in range(2)), torch.zeros(3, dtype=torch.int32, device="cuda"))
    st = torch.zeros((3, 2, 20), device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hyp.attn_token(pr.cache, pr.rule, q, totals=totals, totals_out=into2, out=out, lse=z, workspace=ws)
        hyp.attn_evict(pr.cache, into2, 20, 2, 5, into=small, totals_out=st, kept=kept, workspace=ws)
    for step in range(4):  # the cache grows between replays; every replay is compared with a direct call
        for x in (out, z, into2, kept, st):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, lse = hyp.attn_token(pr.cache, pr.rule, q, totals=totals, totals_out=into)
        assert torch.equal(out, want) and torch.equal(z, lse) and torch.equal(into, into2)
        k2 = hyp.attn_evict(pr.cache, into, 20, 2, 5, into=hyp.AttnCache(torch.zeros_like(small._keep[0]), torch.zeros_like(small._keep[1]), torch.zeros_like(small._keep[2])),
                            totals_out=torch.zeros_like(st))
        assert torch.equal(kept, k2)
        q.mul_(1.1)
        pr.cache._keep[2].sub_(3).clamp_(min=0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_same_bits_from_run_to_run(dtype):
    pr = Problem(24, dtype, 8, 2, 128, held=[700, 333, 5], rows=[200, 333, 5], prefix=300, slopes=True)
    q, start, *_ = pr.device()
    first = hyp.attn_prompt(pr.cache, pr.rule, q, start)
    totals = torch.zeros((3, 2, 700), device="cuda")
    one = hyp.attn_received(pr.cache, pr.rule, q, start, first[1], totals, totals_out=torch.empty_like(totals))
    tok = hyp.attn_token(pr.cache, pr.rule, q[:3])
    for _ in range(3):
        again = hyp.attn_prompt(pr.cache, pr.rule, q, start)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        assert torch.equal(one, hyp.attn_received(pr.cache, pr.rule, q, start, first[1], totals, totals_out=torch.empty_like(totals)))
        assert all(torch.equal(a, b) for a, b in zip(tok, hyp.attn_token(pr.cache, pr.rule, q[:3])))


def test_the_weights_of_a_row_add_up_to_one():
    # a property that needs no reference, at a size that has none: 2000 rows over 4000 keys
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((1, 2, 4000, 128), generator=g, device="cuda").to(BF) for _ in range(2))
    v.fill_(1.0)
    cache = hyp.AttnCache(k, v, torch.tensor([4000], dtype=torch.int32, device="cuda"))
    rule = hyp.AttnRule(0.1, cap=30.0)
    q = torch.randn((2000, 8, 128), generator=g, device="cuda").to(BF)
    start = torch.tensor([0, 2000], dtype=torch.int32, device="cuda")
    out, lse = hyp.attn_prompt(cache, rule, q, start)
    assert float((out.float() - 1).abs().max()) <= 2.0 ** -7
    totals = hyp.attn_received(cache, rule, q, start, lse, torch.zeros((1, 2, 4000), device="cuda"))
    assert float((totals.double().sum(-1) / 8000 - 1).abs().max()) < 1e-5
    totals = hyp.attn_received(cache, rule, q, start, lse, torch.zeros((1, 2, 4000), device="cuda"), last=100)
    assert float((totals.double().sum(-1) / 400 - 1).abs().max()) < 1e-5


def test_refusals():
    pr = Problem(2, BF, 4, 2, 64, held=[20, 20], prefix=10)
    q, start, *_ = pr.device()
    for bad in (dict(q=q[:, :3]), dict(q=q.float()), dict(q=q[:1]), dict(totals=torch.zeros((2, 2, 19), device="cuda")), dict(lse=torch.zeros((2, 4), dtype=BF, device="cuda")),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, hyp.HypError)):
            hyp.attn_token(pr.cache, pr.rule, bad.pop("q", q), **bad)
    with pytest.raises(ValueError):
        hyp.attn_prompt(pr.cache, pr.rule, q, start[:2])
    with pytest.raises(hyp.HypError):
        hyp.attn_prompt(pr.cache, hyp.AttnRule(0.0), q, start)
    with pytest.raises(hyp.HypError):
        hyp.attn_prompt(pr.cache, hyp.AttnRule(1.0, cap=-1.0), q, start)
    with pytest.raises(ValueError):
        hyp.AttnCache(pr.k.cuda(), pr.v.cuda()[:, :, :5], pr.cache._keep[2])
    with pytest.raises(ValueError):
        hyp.AttnCache(pr.k.cuda(), pr.v.cuda(), pr.cache._keep[2].long())
    with pytest.raises(ValueError):
        hyp.AttnCache(pr.k.cuda(), pr.v.cuda(), pr.cache._keep[2], most=1000)
    with pytest.raises(hyp.HypError):
        three = torch.zeros((4, 2, 3, 64), dtype=BF, device="cuda")
        hyp.attn_token(hyp.AttnCache(three, three, pr.cache._keep[2], page_table=torch.zeros((2, 2), dtype=torch.int32, device="cuda")), pr.rule, q)
    with pytest.raises(hyp.HypError):
        hyp.attn_evict(pr.cache, torch.zeros((2, 2, 20), device="cuda"), 5, sink=3, recent=3)
    with pytest.raises(ValueError):
        hyp.attn_received(pr.cache, pr.rule, q, start, torch.zeros((3, 4), device="cuda"), torch.zeros((2, 2, 20), device="cuda"))
