"""mx_token over groups of more than 16 query heads where a wave takes two tiles of them: enough listed blocks, most of which are none, or room for
enough keys, over few keys that the reference has to look at."""
import pytest
import torch

import paper_2511_14450_amd as hyp
from tests.mx_problem import BF, Problem
from tests.test_gpu_mx_token import FORMATS, check, rows
from tests.test_mx_cuts import plan
from tests.test_mx_rules import ask  # noqa: F401

pytestmark = pytest.mark.gpu
HELD = [4200, 70, 0, 4095, 33, 16, 1, 300]


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("group,d", [(17, 128), (24, 64), (32, 96), (33, 32), (71, 80)])
def test_listed_blocks(ask, group, d, formats):  # noqa: F811
    pr = Problem(41, HELD, nkv=1, d=d, formats=formats, dtype=BF, block=256, most=8192).fill()
    listed = 2048 // (8 * -(-group // 32)) + 1
    assert plan(ask, 8, group, listed * 256, page=8192, block=256, features=-(-d // 32))["tiles"] == 2
    q, lists = rows(pr, group, BF), [[[i % 17 if i % 20 == 3 and h else -1 for i in range(listed)]] for h in HELD]
    check(pr, q, lists, cap=20.0, slopes=[0.01 * (h % 5) for h in range(group)])


@pytest.mark.parametrize("formats", FORMATS)
@pytest.mark.parametrize("group,d", [(17, 128), (24, 40), (32, 96), (48, 64)])
def test_all_keys_in_parts_of_pages(ask, group, d, formats):  # noqa: F811
    most = 2048 * 256 // (8 * -(-group // 32)) + 4000
    assert plan(ask, 8, group, most, page=1024, features=-(-d // 32))["tiles"] == 2
    pr = Problem(42, HELD, nkv=1, d=d, formats=formats, dtype=BF, block=0, most=most, layout="pages", page=1024).fill()
    q = rows(pr, group, BF)
    assert hyp.mx_token_workspace_bytes(pr.cache, q.cuda()) > 0
    check(pr, q)
    check(pr, q, cap=20.0, slopes=[0.01 * (h % 5) for h in range(group)])


def test_equal_bits_and_recorded_graphs():
    pr = Problem(43, HELD, nkv=1, d=128, formats=("e4m3", "e2m1"), dtype=BF, block=0, most=70000, layout="pages", page=1024).fill()
    q, rule = rows(pr, 24, BF).cuda(), hyp.AttnRule(0.1, cap=30.0)
    want = hyp.mx_token(pr.cache, rule, q)
    out, lse = torch.zeros_like(q), torch.zeros((8, 24), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hyp.mx_token(pr.cache, rule, q, out=out, lse=lse)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = hyp.mx_token(pr.cache, rule, q)
        assert all(torch.equal(a, b) for a, b in zip((out, lse), want)) and all(torch.equal(a, b) for a, b in zip(again, want))
