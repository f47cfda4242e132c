"""Numbers that do not fit the 32 bits of hyp_attn.h are refused, not cut."""
import pytest
import torch

import paper_2511_14450_amd as hyp

pytestmark = pytest.mark.gpu


def test_numbers_beyond_32_bits():
    key = torch.zeros((1, 1, 1, 8), device="cuda")
    one, start = torch.ones(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    pool = key.expand(1, 1, 1 << 20, 8)
    with pytest.raises((ValueError, hyp.HypError)):  # room for 2^32 + 2^20 keys
        hyp.AttnCache(pool, pool, one, page_table=torch.zeros((1, 4097), dtype=torch.int32, device="cuda"))
    with pytest.raises((ValueError, hyp.HypError)):
        hyp.AttnCache(key.expand(1, 1, (1 << 32) + 5, 8), key.expand(1, 1, (1 << 32) + 5, 8), one)
    long = key[0].expand(1, (1 << 32) + 5, 8)
    with pytest.raises((ValueError, hyp.HypError)):
        hyp.AttnCache(key, key, one, prefix_k=long, prefix_v=long)
    cache, rule, q = hyp.AttnCache(key, key, one), hyp.AttnRule(1.0), key[0]
    totals, lse = torch.zeros((1, 1, 1), device="cuda"), torch.zeros((1, 1), device="cuda")
    with pytest.raises((ValueError, hyp.HypError)):
        hyp.attn_received(cache, rule, q, start, lse, totals, last=(1 << 32) + 1)
    for kw in (dict(sink=1 << 32), dict(recent=1 << 32)):
        with pytest.raises((ValueError, hyp.HypError)):
            hyp.attn_evict(cache, totals, 1, **kw)
