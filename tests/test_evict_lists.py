"""Eviction with lists of no entries: their counts are zeros, whoever made the array."""
import ctypes

import numpy as np
import pytest
import torch

from conftest import gpu_available
from pages_ref import Host
from test_abi_cpu import FAKE, _desc

wk = pytest.importorskip("paper_2609_38121_amd")
from paper_2609_38121_amd import _lib  # noqa: E402


def ints(*shape, **kw):
    return torch.full(shape, 77, dtype=torch.int32, **kw)


@pytest.mark.parametrize("kw", [{}, {"max_sel": 0}])
def test_counts_reach_the_library(kw, monkeypatch):
    c = wk.WushKVCache(3, 2, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=500, device="cpu")
    pool, weights, real, seen = wk.WushKVPool(c), torch.zeros(3, 2, c.max_pages), _lib.lib(), []

    class Library:
        def __getattr__(self, name):
            return (lambda *args: seen.append(args) or 0) if name == "wushkv_evict_pages" else getattr(real, name)

    monkeypatch.setattr(wk, "_launch_stream", lambda dev, stream: 0)
    monkeypatch.setattr(_lib, "lib", Library)
    if not kw:
        kw = {"sel": ints(3, 2, 0)}
    for given in (None, ints(3, 2)):
        sel, n_sel, _ = wk.wushkv_evict_pages(c, pool, weights, ints(3), n_sel=given, **kw)
        assert sel.shape == (3, 2, 0) and seen[-1][8] == n_sel.data_ptr() != 0 and seen[-1][9] == 0
        assert given is None or n_sel is given
    for wrong in (ints(3), ints(3, 2).long(), ints(2, 3).t()):
        with pytest.raises(ValueError):
            wk.wushkv_evict_pages(c, pool, weights, ints(3), n_sel=wrong, **kw)


@pytest.mark.skipif(gpu_available(), reason="fake device pointers: run only where no GPU exists")
def test_no_list_where_there_are_no_entries():
    def evict(sel, n_sel, width):
        return _lib.lib().wushkv_evict_pages(ctypes.byref(_desc()), ctypes.byref(_lib.PoolDesc(FAKE, FAKE, FAKE)), FAKE, FAKE, 0,
                                             FAKE, FAKE, sel, n_sel, width, FAKE, None)
    # (past the checks there is no device to launch on)
    assert evict(None, FAKE, 0) == evict(FAKE, FAKE, 0) == evict(None, None, 0) == _lib.ELAUNCH
    assert evict(None, FAKE, 1) == evict(FAKE, None, 0) == evict(None, FAKE + 4, 0) == _lib.EINVAL


@pytest.mark.gpu
def test_counts_are_zeros(gpu):
    h = Host(np.random.default_rng(1), [700, 500, 30], 2, 64, 2)
    for given in (None, ints(3, 2, device=gpu)):
        c, pool = h.cache(gpu)
        weights, budget = torch.ones(3, 2, h.max_pages, device=gpu), torch.full((3,), 4, dtype=torch.int32, device=gpu)
        for table_out in (None, torch.empty_like(c.page_table)):
            sel, n_sel, gone = wk.wushkv_evict_pages(c, pool, weights, budget, n_sel=given, max_sel=0, table_out=table_out,
                                                     refs_out=None if table_out is None else torch.empty_like(pool.refs))
            assert sel.shape == (3, 2, 0) and (n_sel == 0).all()
            # (in place first: after it there is nothing more to evict)
            want = [h.complete(b) - 4 if table_out is None and h.complete(b) > 4 else 0 for b in range(3)]
            assert gone.tolist() == want


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[700, 500, 30]])
def test_a_pool_of_no_pages(gpu, lens):
    """Nothing leaves, and the new table is the old one."""
    h = Host(np.random.default_rng(2), lens, 2, 64, 2)
    c = wk.WushKVCache(3, 2, 64, 2, h.s_sink, h.s_keep, h.s_flush, 0.96, 0.92, max_seq_len=800, win_slots=h.win_slots,
                       page_order="none", n_pages=0, device=gpu)
    c.seq_len.copy_(torch.from_numpy(h.seq_len))
    c.quant_end.copy_(torch.from_numpy(h.quant_end))
    pool = wk.WushKVPool(c)
    c.page_table[1, 2] = 3
    pool.held.fill_(5)
    at = torch.empty(4, dtype=torch.int32, device=gpu)  # (arrays of no elements have no address)
    desc = _lib.PoolDesc(at.data_ptr(), pool.held.data_ptr(), pool.low.data_ptr())
    weights, budget, table = torch.ones(3, 2, c.max_pages, device=gpu), torch.zeros(3, dtype=torch.int32, device=gpu), \
        torch.full_like(c.page_table, 55)
    sel, n_sel, gone = ints(3, 2, 4, device=gpu), ints(3, 2, device=gpu), ints(3, device=gpu)
    assert _lib.lib().wushkv_evict_pages(
        ctypes.byref(c.desc), ctypes.byref(desc), weights.data_ptr(), budget.data_ptr(), 0, table.data_ptr(), at.data_ptr(),
        sel.data_ptr(), n_sel.data_ptr(), 4, gone.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(table, c.page_table)
    assert (sel == -1).all() and (n_sel == 0).all() and (gone == 0).all()
