"""Calls of hyp_mx.h in recorded graphs, replayed between eager work on other inputs, on other streams, and two graphs that share a workspace."""
import pytest
import torch

import paper_2511_14450_amd as hyp
from tests.mx_problem import BF, F32, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_step_of_generation_in_a_graph(dtype):
    # lens grows on the device; one side by replays, the other by calls
    n, nkv, heads, d, most = 3, 2, 8, 128, 1500
    sides = []
    for _ in range(2):
        pr = Problem(1, [900, 1200, 40], nkv=nkv, d=d, block=32, dtype=dtype, layout="pages", page=64, most=most, formats=("e4m3", "e2m1")).fill()
        sides.append(dict(pr=pr, k=torch.zeros((n, nkv, d), dtype=dtype, device="cuda"), v=torch.zeros((n, nkv, d), dtype=dtype, device="cuda"), q=torch.zeros((n, heads, d), dtype=dtype, device="cuda"),
                          blocks=torch.zeros((n, nkv, 20), dtype=torch.int32, device="cuda"), out=torch.zeros((2, n, heads, d), dtype=dtype, device="cuda"), lse=torch.zeros((2, n, heads), device="cuda"),
                          read=[torch.zeros((n, nkv, 64, d), dtype=dtype, device="cuda") for _ in range(2)]))
    rule = hyp.AttnRule(d ** -0.5, cap=30.0)
    pr = sides[0]["pr"]
    need = max(hyp.mx_token_workspace_bytes(pr.cache, sides[0]["q"]), hyp.mx_token_workspace_bytes(pr.cache, sides[0]["q"], 20), hyp.mx_select_workspace_bytes(pr.cache, sides[0]["q"], 20), 16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(s):
        c = s["pr"].cache
        s["pr"].lens.add_(1)
        hyp.mx_write(c, s["k"], s["v"])
        hyp.mx_select(c, s["q"], 20, sink=1, recent=2, blocks=s["blocks"], workspace=ws)
        hyp.mx_token(c, rule, s["q"], blocks=s["blocks"], out=s["out"][0], lse=s["lse"][0], workspace=ws)
        hyp.mx_token(c, rule, s["q"], out=s["out"][1], lse=s["lse"][1], workspace=ws)
        hyp.mx_read(c, *s["read"], first=s["pr"].lens - 60)

    lens = sides[0]["pr"].lens.clone()
    step(sides[0])
    torch.cuda.synchronize()
    sides[0]["pr"].fill()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sides[0])
    assert torch.equal(sides[0]["pr"].lens, lens)  # recording ran nothing
    g = torch.Generator().manual_seed(2)
    for turn in range(40):
        for name in ("k", "v", "q"):
            x = torch.randn(sides[0][name].shape, generator=g).to(dtype)
            for s in sides:
                s[name].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)
        step(sides[1])
        for name in ("blocks", "out", "lse"):
            assert torch.equal(sides[0][name], sides[1][name]), (turn, name)
        assert all(torch.equal(a, b) for a, b in zip(sides[0]["read"], sides[1]["read"]))
        assert torch.equal(sides[0]["pr"].lens, sides[1]["pr"].lens)
    a, b = (s["pr"] for s in sides)
    for x, y in ((a.lo, b.lo), (a.hi, b.hi)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_prompts_of_changing_lengths_in_a_graph():
    pr = Problem(3, [80, 80], d=64, block=16, most=80)
    k, v = (torch.zeros((90, 2, 64), device="cuda") for _ in range(2))
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    pr.write([0, 0], [1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hyp.mx_write(pr.cache, k, v, q_start=start)
    other = Problem(3, [80, 80], d=64, block=16, most=80)
    g = torch.Generator().manual_seed(4)
    for lens, counts in (([40, 3], [40, 3]), ([50, 60], [10, 57]), ([51, 60], [1, 0]), ([80, 80], [29, 20]), ([7, 80], [7, 80])):
        k.copy_(torch.randn(k.shape, generator=g))
        v.copy_(torch.randn(v.shape, generator=g))
        for p in (pr, other):
            p.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        start.copy_(torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        hyp.mx_write(other.cache, k, v, q_start=start)
        for b, n in enumerate(lens):
            assert torch.equal(pr.k[b, :, :n], other.k[b, :, :n]) and torch.equal(pr.vs[b, :, :, :n], other.vs[b, :, :, :n])
            blocks = -(-n // 16)
            assert torch.equal(pr.lo[b, :, :blocks], other.lo[b, :, :blocks]) and torch.equal(pr.hi[b, :, :blocks], other.hi[b, :, :blocks])


def test_calls_on_streams_of_their_own():
    # each stream with a cache and a workspace of its own; what a call returns is made on its stream
    prs = [Problem(5 + i, [2000, 900], nkv=2, d=128, dtype=BF, block=16).fill() for i in range(3)]
    qs = [torch.randn((2, 8, 128), generator=pr.gen).to(BF).cuda() for pr in prs]
    rule = hyp.AttnRule(0.1)
    want = [(hyp.mx_select(pr.cache, q, 5, recent=1), *hyp.mx_token(pr.cache, rule, q)) for pr, q in zip(prs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in prs]
    for _ in range(5):
        got = [(hyp.mx_select(pr.cache, q, 5, recent=1, stream=s), *hyp.mx_token(pr.cache, rule, q, stream=s)) for pr, q, s in zip(prs, qs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_two_graphs_that_share_a_workspace():
    prs = [Problem(9 + i, [3000, 1500], nkv=2, d=64, dtype=F32).fill() for i in range(2)]
    qs = [torch.randn((2, 4, 64), generator=pr.gen).cuda() for pr in prs]
    rule = hyp.AttnRule(0.125)
    want = [hyp.mx_token(pr.cache, rule, q) for pr, q in zip(prs, qs)]
    need = hyp.mx_token_workspace_bytes(prs[0].cache, qs[0])
    assert need > 0
    ws, graphs, outs = torch.empty(need, dtype=torch.uint8, device="cuda"), [], []
    for pr, q in zip(prs, qs):
        out, lse = torch.zeros_like(q), torch.zeros((2, 4), device="cuda")
        hyp.mx_token(pr.cache, rule, q, out=out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            hyp.mx_token(pr.cache, rule, q, out=out, lse=lse, workspace=ws)
        outs.append((out, lse))
    for turn in range(6):
        for i in ((0, 1), (1, 0), (0, 0))[turn % 3]:
            outs[i][0].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1]) for i in range(2) if turn % 3 < 2 or i == 0)


def test_the_widest_heads_are_recorded_without_a_call_before():
    # sixteen heads of 256 features join in more LDS than a launch has by itself
    pr = Problem(13, [100], nkv=1, d=256, formats=("e2m1", "e4m3"), dtype=F32).fill()
    q, out, lse = torch.randn((1, 16, 256), generator=pr.gen).cuda(), torch.zeros((1, 16, 256), device="cuda"), torch.zeros((1, 16), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hyp.mx_token(pr.cache, hyp.AttnRule(0.0625), q, out=out, lse=lse)
    graph.replay()
    torch.cuda.synchronize()
    want = hyp.mx_token(pr.cache, hyp.AttnRule(0.0625), q)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
