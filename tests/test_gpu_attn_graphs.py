"""Calls of hyp_attn.h in a recorded graph, replayed between eager work on other inputs: prompts in one part and in several, the weight their keys
receive in both forms, single tokens, eviction in place."""
import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import attn_received_cases as cases
from tests.test_gpu_attn import BF, F32, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form", ["parts", "one part", "pairs of blocks"])
def test_prompts_in_a_graph(dtype, form):
    pr = {"parts": lambda: Problem(51, dtype, 4, 2, 64, held=[1500, 40], rows=[3, 40], prefix=200, slopes=True),
          "one part": lambda: Problem(52, dtype, 8, 2, 128, held=[300, 41, 7], rows=[300, 30, 7], prefix=20, docs=3),
          "pairs of blocks": lambda: cases.problem(cases.case(rule=dict(cap=20.0)), dtype, Problem)}[form]()
    q, start, q_pos, q_doc, see = pr.device()
    n = len(pr.held)
    ws = torch.empty(max(hyp.attn_workspace_bytes(pr.cache, pr.rule, q, start), 16), dtype=torch.uint8, device="cuda")
    totals = torch.rand((n, pr.nkv, pr.most), device="cuda")

    def calls(out, lse, got):
        hyp.attn_prompt(pr.cache, pr.rule, q, start, q_pos=q_pos, q_doc=q_doc, out=out, lse=lse, workspace=ws)
        hyp.attn_received(pr.cache, pr.rule, q, start, lse, totals, q_pos=q_pos, q_doc=q_doc, totals_out=got)

    recorded, eager = ([torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda"), torch.zeros_like(totals)] for _ in range(2))
    calls(*recorded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(*recorded)
    for _ in range(4):
        for t in recorded + eager:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)
        calls(*eager)
        assert all(torch.equal(a, b) for a, b in zip(recorded, eager))
        q.mul_(1.1)
        totals.add_(0.5)


def test_tokens_and_eviction_in_place_in_a_graph():
    # a cache that a step fills and that is then cut back, as a server would record it: one side by replays, the other by calls
    g = torch.Generator().manual_seed(6)
    n, nkv, d, room, keep = 3, 2, 64, 40, 24
    make = lambda: dict(k=torch.zeros((n, nkv, room, d), device="cuda"), v=torch.zeros((n, nkv, room, d), device="cuda"), lens=torch.zeros(n, dtype=torch.int32, device="cuda"),  # noqa: E731
                        pos=torch.zeros((n, nkv, room), dtype=torch.int32, device="cuda"), totals=torch.zeros((n, nkv, room), device="cuda"),
                        kept=torch.zeros((n, nkv, keep), dtype=torch.int32, device="cuda"), out=torch.zeros((n, 4, d), device="cuda"), lse=torch.zeros((n, 4), device="cuda"))
    sides = [make(), make()]
    rule, now, q = hyp.AttnRule(0.125, slopes=torch.tensor([0.01, 0.02, 0.03, 0.04]).cuda()), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros((n, 4, d), device="cuda")
    caches = [hyp.AttnCache(s["k"], s["v"], s["lens"], key_pos=s["pos"]) for s in sides]
    need = max(hyp.attn_workspace_bytes(caches[0], rule, q, totals=True), hyp.attn_evict_workspace_bytes(caches[0], keep))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(s, cache):
        hyp.attn_token(cache, rule, q, q_pos=now, totals=s["totals"], out=s["out"], lse=s["lse"], workspace=ws)
        hyp.attn_evict(cache, s["totals"], keep, sink=1, recent=4, now=now, kept=s["kept"], workspace=ws)

    step(sides[1], caches[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sides[0], caches[0])
    for s in sides:
        for t in s.values():
            t.zero_()
    for turn in range(60):
        key, value = torch.randn((n, nkv, d), generator=g).cuda(), torch.full((n, nkv, d), float(turn), device="cuda")
        for s in sides:
            for b in range(n):  # a key more in each turn, three in some of a request's
                for _ in range(3 if (turn + b) % 3 == 0 else 1):
                    x = int(s["lens"][b])
                    s["k"][b, :, x], s["v"][b, :, x], s["pos"][b, :, x], s["totals"][b, :, x] = key[b], value[b], turn, 0.0
                    s["lens"][b] += 1
        now.fill_(turn + 1)
        q.copy_(torch.randn((n, 4, d), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        step(sides[1], caches[1])
        for name in sides[0]:
            assert torch.equal(sides[0][name], sides[1][name]), (turn, name)
        assert int(sides[0]["lens"].max()) <= keep
