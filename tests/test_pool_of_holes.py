"""A pool made from a cache whose rows have holes (evicted pages): the pages behind a
hole are held, and a hole among the quantised positions is given no page."""
import numpy as np
import pytest
import torch

import pages_ref
from pages_ref import Host

wk = pytest.importorskip("paper_2609_38121_amd")


def test_held_reaches_behind_holes():
    c = wk.WushKVCache(6, 1, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=4 + 64 * 5, page_order="none", n_pages=20, device="cpu")
    rows = [[3, -1, 5, -1, -1],   # a hole in the midst
            [-1, -1, 7, 8, 9],    # at the start
            [1, 2, 4, -1, -1],    # behind the last page, where positions are
            [-1, -1, -1, -1, -1],  # every page has left
            [-1, -1, -1, -1, -1],  # nothing yet
            [3, 10, 20, -2, -1]]  # entries outside the pool; pages ahead of the positions
    c.page_table.copy_(torch.tensor(rows))
    c.seq_len.copy_(torch.tensor([300, 400, 300, 140, 1, 9]))
    c.quant_end.copy_(torch.tensor([4 + 64 * 3, 4 + 64 * 4 + 1, 4 + 64 * 4, 4 + 65, 0, 0]))
    pool = wk.WushKVPool(c)
    assert pool.held.dtype is torch.int32 and pool.held.tolist() == [3, 5, 4, 2, 0, 2]
    assert pool.refs.tolist() == [0, 1, 1, 2, 1, 1, 0, 1, 1, 1, 1] + [0] * 9
    # as before where there is no hole
    full = wk.WushKVCache(2, 1, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=4 + 64 * 5, device="cpu")
    assert wk.WushKVPool(full).held.tolist() == [5, 5]


@pytest.mark.gpu
def test_a_new_pool_after_an_eviction(gpu):
    """Sequences go on from a new pool as from the one that they had."""
    rng = np.random.default_rng(9)
    h = Host(rng, [700, 64 * 5 + 36, 333, 20], 2, 64, 2, max_pages=14, spare=20)
    c, pool = h.cache(gpu)
    weights = rng.standard_normal((4, 2, 14)).astype(np.float32)
    weights[1, :, 3:] = -9.0  # (the last of them, so that its row ends with a hole)
    budget = np.full(4, 2, np.int32)
    wk.wushkv_evict_pages(c, pool, torch.from_numpy(weights).to(gpu), torch.from_numpy(budget).to(gpu))
    pages_ref.evict(h, weights, budget, 0, 14)
    new = wk.WushKVPool(c)
    assert torch.equal(new.refs, pool.refs) and torch.equal(new.held, pool.held)
    reach = h.seq_len + 100
    status = wk.wushkv_assign_pages(c, new, reach=torch.from_numpy(reach.astype(np.int32)).to(gpu))
    assert np.array_equal(status.cpu().numpy(), pages_ref.assign(h, reach=reach))
    assert np.array_equal(c.page_table.cpu().numpy(), h.table) and np.array_equal(new.refs.cpu().numpy(), h.refs)
