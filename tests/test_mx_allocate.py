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


@pytest.mark.parametrize("block_keys,page_keys", [(24, 0), (24, 32), (48, 128), (64, 32), (8, 32), (-16, 0), (8192, 0)])
def test_blocks_of_another_size_than_was_asked_for_are_not_made(block_keys, page_keys):
    # a page of 32 keys with room for one block of 24 had one of 32, one of 128 with room for two of 48 had two of 64
    with pytest.raises(ValueError, match="block_keys"):
        mx.MxCache.allocate(3, 2, 60, 64, block_keys=block_keys, page_keys=page_keys, device="cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("block_keys,page_keys", [(0, 0), (16, 0), (4096, 0), (16, 32), (32, 32), (64, 256)])
def test_blocks_have_the_size_that_was_asked_for(block_keys, page_keys):
    assert mx.MxCache.allocate(3, 2, 60, 64, block_keys=block_keys, page_keys=page_keys).block_keys == block_keys
