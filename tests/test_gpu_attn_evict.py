"""Eviction (hyp_attn.h) against its rule on the host: ties, numbers that are none, what is always kept, in place and into another
cache, pages, lengths."""
import math

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import attn_reference as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def build(seed, dtype, held, nkv, d, prefix=0, page=0, pos=False, doc=False, totals="heavy", room=None):
    g = torch.Generator().manual_seed(seed)
    n, room = len(held), room or max(held + [1])
    k, v = (torch.randn((n, nkv, room, d), generator=g).to(dtype) for _ in range(2))
    t = torch.randn((n, nkv, room), generator=g).mul(2).exp()
    if totals == "ties":
        t = torch.randint(0, 3, (n, nkv, room), generator=g).float()
        t[t == 0] *= -1.0  # -0 and 0 are the same weight
    elif totals == "odd":
        kind = torch.randint(0, 7, t.shape, generator=g)
        for x, value in enumerate((math.nan, math.inf, -math.inf, -1.0, 0.0)):
            t[kind == x] = value
    elif totals == "equal":
        t.fill_(0.25)
    key_pos = torch.stack([torch.stack([torch.randperm(3 * room, generator=g)[:room] for _ in range(nkv)]) for _ in range(n)]).int() if pos else None
    key_doc = torch.randint(-1, 5, (n, nkv, room), generator=g, dtype=torch.int32) if doc else None
    pre = torch.zeros((nkv, prefix, d), dtype=dtype) if prefix else None
    table = None
    if page:
        pages = -(-room // page)
        table = torch.randperm(n * pages, generator=g).reshape(n, pages).int()
    return g, k, v, t, key_pos, key_doc, pre, table


def pooled(x, table, page):
    n, nkv, room, d = x.shape
    pages = table.shape[1]
    full = torch.zeros((n, nkv, pages * page, d), dtype=x.dtype)
    full[:, :, :room] = x
    pool = torch.zeros((n * pages, nkv, page, d), dtype=x.dtype)
    pool[table.reshape(-1).long()] = full.reshape(n, nkv, pages, page, d).permute(0, 2, 1, 3, 4).reshape(-1, nkv, page, d)
    return pool


def unpooled(pool, table):
    n, pages = table.shape
    return pool[table.long()].transpose(1, 2).reshape(n, pool.shape[1], pages * pool.shape[2], pool.shape[3])


def check(dtype, held, nkv, d, keep, sink=0, recent=0, now=None, **more):
    page, prefix = more.get("page", 0), more.get("prefix", 0)
    g, k, v, t, key_pos, key_doc, pre, table = build(sum(held) + keep, dtype, held, nkv, d, **more)
    n, room = len(held), k.shape[2]
    want = torch.empty((n, nkv, keep), dtype=torch.int32)
    for b in range(n):
        for c in range(nkv):
            pos = key_pos[b, c].tolist() if key_pos is not None else [prefix + j for j in range(room)]
            want[b, c] = torch.tensor(ref.evict(t[b, c].tolist(), held[b], keep, sink, recent, pos, prefix, prefix + held[b] if now is None else now[b]))
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    now_d = None if now is None else torch.tensor(now, dtype=torch.int32).cuda()
    valid = want >= 0
    safe = want.clamp(min=0).long()
    pick = lambda x: x.gather(2, safe)  # noqa: E731
    pick_rows = lambda x: x.gather(2, safe[..., None].expand(-1, -1, -1, d))  # noqa: E731
    src_k, src_v = (pooled(k, table, page).cuda(), pooled(v, table, page).cuda()) if page else (k.cuda(), v.cuda())
    pos_full = key_pos if key_pos is not None else (prefix + torch.arange(room, dtype=torch.int32)).expand(n, nkv, room)

    # into another cache, with room to spare
    cache = hyp.AttnCache(src_k, src_v, torch.tensor(held, dtype=torch.int32).cuda(), page_table=dev(table), most=room, prefix_k=dev(pre), prefix_v=dev(pre),
                          key_pos=dev(key_pos), key_doc=dev(key_doc))
    to_k, to_v = (torch.full((n, nkv, keep + 2, d), 5.0, dtype=dtype, device="cuda") for _ in range(2))
    to_len, to_pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.full((n, nkv, keep + 2), -9, dtype=torch.int32, device="cuda")
    to_doc, to_t = torch.full_like(to_pos, -9), torch.full((n, nkv, keep + 2), -9.0, device="cuda")
    to = hyp.AttnCache(to_k, to_v, to_len, key_pos=to_pos, key_doc=to_doc)
    td = t.cuda()
    kept = hyp.attn_evict(cache, td, keep, sink, recent, now=now_d, into=to, totals_out=to_t)
    assert torch.equal(kept.cpu(), want)
    assert to_len.tolist() == [min(h, keep) for h in held]
    vm = valid[..., None].expand(-1, -1, -1, d)
    for got, x in ((to_k, k), (to_v, v)):
        got = got.cpu()
        assert torch.equal(got[:, :, :keep][vm], pick_rows(x)[vm]) and bool((got[:, :, :keep][~vm] == 5).all()) and bool((got[:, :, keep:] == 5).all())
    bits = lambda x: x.contiguous().view(torch.int32)  # noqa: E731
    assert torch.equal(bits(to_t.cpu()[:, :, :keep])[valid], bits(pick(t))[valid]) and bool((to_t.cpu()[:, :, :keep][~valid] == -9).all())
    assert torch.equal(to_pos.cpu()[:, :, :keep][valid], pick(pos_full)[valid])
    doc_want = pick(key_doc)[valid] if key_doc is not None else torch.full((int(valid.sum()),), -1, dtype=torch.int32)
    assert torch.equal(to_doc.cpu()[:, :, :keep][valid], doc_want)

    # in place: the same keys in the same slots
    pos_d, doc_d = dev(key_pos), dev(key_doc)
    src_k, src_v, lens = src_k.clone(), src_v.clone(), torch.tensor(held, dtype=torch.int32).cuda()
    cache = hyp.AttnCache(src_k, src_v, lens, page_table=dev(table), most=room, prefix_k=dev(pre), prefix_v=dev(pre), key_pos=pos_d, key_doc=doc_d)
    kept = hyp.attn_evict(cache, td, keep, sink, recent, now=now_d)
    assert torch.equal(kept.cpu(), want) and lens.tolist() == [min(h, keep) for h in held]
    for got, x in ((src_k, k), (src_v, v)):
        got = unpooled(got.cpu(), table) if page else got.cpu()
        m = min(keep, got.shape[2])
        assert torch.equal(got[:, :, :m][vm[:, :, :m]], pick_rows(x)[:, :, :m][vm[:, :, :m]])
    m = min(keep, room)
    assert torch.equal(bits(td.cpu()[:, :, :m])[valid[..., :m]], bits(pick(t))[:, :, :m][valid[..., :m]])
    if key_pos is not None:
        assert torch.equal(pos_d.cpu()[:, :, :m][valid[..., :m]], pick(key_pos)[:, :, :m][valid[..., :m]])
    if key_doc is not None:
        assert torch.equal(doc_d.cpu()[:, :, :m][valid[..., :m]], pick(key_doc)[:, :, :m][valid[..., :m]])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("held,nkv,d,keep", [([96, 70], 2, 64, 64), ([1, 0, 5], 1, 128, 3), ([200], 3, 80, 1), ([1025, 1024, 1023], 2, 40, 1023),
                                             ([3000, 2999, 77], 2, 128, 1500), ([40, 50], 2, 33, 20), ([10, 20], 1, 64, 30)])
def test_lengths_and_heads(dtype, held, nkv, d, keep):
    check(dtype, held, nkv, d, keep, sink=min(2, keep // 3), recent=keep // 3)


@pytest.mark.parametrize("totals", ["ties", "odd", "equal"])
@pytest.mark.parametrize("keep", [7, 64, 100, 149])
def test_ties_and_numbers_that_are_none(totals, keep):
    check(BF, [150, 131, keep], 2, 64, keep, sink=1, recent=3, totals=totals)


@pytest.mark.parametrize("page", [0, 16, 128])
def test_positions_ids_and_pages(page):
    check(BF, [300, 211, 30], 2, 64, 128, sink=4, recent=20, prefix=33, page=page, pos=True, doc=True, now=[900, 450, 5])
    check(F32, [300, 211, 30], 2, 64, 128, sink=4, recent=20, prefix=33, page=page, doc=True)


def test_a_long_request():
    check(BF, [40000], 1, 8, 17000, sink=4, recent=4000)
    check(BF, [40000], 1, 8, 17000, totals="ties")


def test_sink_and_recent_take_the_whole_budget():
    check(BF, [100, 64], 2, 64, 16, sink=6, recent=10)
    check(BF, [100, 64], 2, 64, 16, recent=16)


def test_evicting_what_was_evicted():
    # a cache that grows by a key a step and is cut back each time: totals, positions and keys stay together
    g = torch.Generator().manual_seed(5)
    n, nkv, d, room, keep = 2, 2, 64, 24, 16
    k, v = (torch.zeros((n, nkv, room, d), device="cuda") for _ in range(2))
    lens, pos, totals = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros((n, nkv, room), dtype=torch.int32, device="cuda"), torch.zeros((n, nkv, room), device="cuda")
    cache, rule = hyp.AttnCache(k, v, lens, key_pos=pos), hyp.AttnRule(0.125, slopes=torch.tensor([0.01, 0.02, 0.03, 0.04]).cuda())
    model = [[{"pos": [], "t": []} for _ in range(nkv)] for _ in range(n)]
    for step in range(60):
        at = lens[0].item()
        k[:, :, at], v[:, :, at] = torch.randn((n, nkv, d), generator=g).cuda(), float(step)
        pos[:, :, at], totals[:, :, at] = step, 0.0
        lens += 1
        q = torch.randn((n, 4, d), generator=g).cuda()
        hyp.attn_token(cache, rule, q, q_pos=torch.full((n,), step, dtype=torch.int32, device="cuda"), totals=totals)
        for b in range(n):
            for c in range(nkv):
                model[b][c]["pos"].append(step)
                model[b][c]["t"] = totals[b, c, :at + 1].tolist()
        if at + 1 == room:
            hyp.attn_evict(cache, totals, keep, sink=1, recent=4, now=torch.full((n,), step + 1, dtype=torch.int32, device="cuda"))
            for b in range(n):
                for c in range(nkv):
                    m = model[b][c]
                    slots = ref.evict(m["t"], room, keep, 1, 4, m["pos"], 0, step + 1)
                    m["pos"], m["t"] = [m["pos"][s] for s in slots], [m["t"][s] for s in slots]
        now = lens[0].item()
        for b in range(n):
            for c in range(nkv):
                assert pos[b, c, :now].tolist() == model[b][c]["pos"] and totals[b, c, :now].tolist() == model[b][c]["t"]
                assert v[b, c, :now, 0].tolist() == [float(p) for p in model[b][c]["pos"]]
