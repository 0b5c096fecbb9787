"""GPU: calls of the cache that fail on the way leave it, and its block manager, as they were."""
import pytest
import torch

import paper_2609_34380_b200 as dps
from paper_2609_34380_b200 import sum_manager as sm
from paper_2609_34380_b200.kv_cache import PagedKvCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_an_extend_that_fails_takes_no_blocks():
    """A step of more rows than the device has memory for: the blocks go back, and the next step takes them and enters them in the table."""
    mgr = sm.SumManager(2, 4, 1)
    cache = PagedKvCache(mgr, 1, 4, 4, 64, 16, max_requests=2, max_tokens_per_request=64)
    cache.admit(), cache.admit()
    assert cache.extend([5, 17]).lengths.tolist() == [5, 17]
    held, table = [list(h) for h in cache.held], cache.block_table.clone()
    with pytest.raises(RuntimeError):
        cache.extend([30, 1], rows=1 << 45)
    mgr.check()
    assert cache.held == held and cache.lengths == [5, 17] and mgr.kv_blocks_in_use == 3 and torch.equal(cache.block_table, table)
    step = cache.extend([30, 1])
    assert step.lengths.tolist() == [35, 18] == cache.lengths and dps.dps_stream_status() == dps.DPS_OK
    assert bool((step.slots >= 0).all()) and len(set(step.slots.tolist())) == 31
    for row, blocks in enumerate(cache.held):
        assert cache.block_table[row, :len(blocks)].tolist() == [u * 4 + i for u, i in blocks]
    cache.finish(0), cache.finish(0)
    mgr.check()
    assert mgr.kv_blocks_in_use == 0
