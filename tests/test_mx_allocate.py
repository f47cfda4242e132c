"""MxCache.allocate: pools of fewer pages than its own table would name."""
import pytest
import torch

from paper_2511_14450_amd import mx


@pytest.mark.parametrize("n_pages", [-1, 0, 5])
def test_a_pool_that_does_not_hold_all_requests_needs_a_table(n_pages):
    # three requests of up to 60 keys have two pages of 32 each; pages outside the pool are cut to its last one, which requests would share
    with pytest.raises(ValueError, match="n_pages.*page_table"):
        mx.MxCache.allocate(3, 2, 60, 64, page_keys=32, n_pages=n_pages, device="cpu")


@pytest.mark.gpu
def test_pools_with_room_for_all_and_tables_of_the_callers():
    assert mx.MxCache.allocate(3, 2, 60, 64, page_keys=32).page_table.tolist() == [[0, 1], [2, 3], [4, 5]]
    more = mx.MxCache.allocate(3, 2, 60, 64, page_keys=32, n_pages=8)
    assert more.k.shape[0] == 8 and more.page_table.tolist() == [[0, 1], [2, 3], [4, 5]]
    table = torch.tensor([[0, 1], [2, 2], [3, 3]], dtype=torch.int32, device="cuda")
    few = mx.MxCache.allocate(3, 2, 60, 64, page_keys=32, n_pages=4, page_table=table)
    assert few.k.shape[0] == 4 and few.page_table is table
