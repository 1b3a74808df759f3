"""Compactions of pools of several blocks of 4096 references, in place and into
other arrays, against the plain form, value for value; pages shared by rows and
held by the caller, boxes that move along.  Another stream keeps the device busy,
so that the workgroups of a launch do not all start together."""
import copy

import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
from gpu_harness import say
from test_pages_schedules_cpu import pool_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages,share", [(4096, 0.4), (8192, 0.5), (9000, 0.95), (20011, 0.3), (32768, 0.9), (32769, 0.5),
                                           (40011, 0.6)])
def test_compaction_of_large_pools(gpu, n_pages, share):
    say("compaction of %d pages, %.2f in use" % (n_pages, share))
    rng = np.random.default_rng([n_pages, 3])
    h = pool_of(rng, n_pages, share)
    codes = rng.integers(-128, 128, (n_pages, 1, 2, 64), np.int8)
    scales = rng.random((1, n_pages), np.float32)
    want, wcodes, wscales = copy.deepcopy(h), codes.copy(), scales.copy()
    live = pages_ref.compact(want, wcodes, wscales)
    c = wk.WushKVCache(h.b, 1, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=4 + 64 * h.max_pages, win_slots=64, page_order="none",
                       n_pages=n_pages, device=gpu)
    pool, bounds = wk.WushKVPool(c), wk.WushKVBounds(c)
    other, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device=gpu)
    put = lambda t, a: t.copy_(torch.from_numpy(np.ascontiguousarray(a).reshape(t.shape)))  # noqa: E731
    for in_place in (True, False, True):
        put(c.pages, h.pages)
        put(c.page_table, h.table)
        put(pool.refs, h.refs)
        put(pool.held, h.held)
        put(bounds.codes, codes)
        put(bounds.scales, scales)
        table, refs = (None, None) if in_place else (torch.empty_like(c.page_table), torch.empty_like(pool.refs))
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(4):
                busy = torch.tanh(busy @ busy)
        t, r, n = wk.wushkv_compact_pages(c, pool, bounds=bounds, table_out=table, refs_out=refs)
        torch.cuda.synchronize()
        assert int(n[0]) == live
        assert np.array_equal(t.cpu().numpy(), want.table) and np.array_equal(r.cpu().numpy(), want.refs)
        assert np.array_equal(c.pages.cpu().numpy(), want.pages.reshape(-1))
        assert np.array_equal(bounds.codes.cpu().numpy(), wcodes) and np.array_equal(bounds.scales.cpu().numpy(), wscales)
        if not in_place:
            assert np.array_equal(c.page_table.cpu().numpy(), h.table) and np.array_equal(pool.refs.cpu().numpy(), h.refs)


def test_arrays_of_a_compaction_swapped_in(gpu):
    """The new table and references put in the old ones' place, twice in turn, with
    calls on them in between."""
    rng = np.random.default_rng(11)
    h = pages_ref.Host(rng, [600, 333, 0, 90], 2, 64, 2, spare=9, max_pages=12)
    c, pool = h.cache(gpu)
    for step in range(3):
        old = c.page_table, pool.refs
        source = np.arange(4)
        source[step % 2] = -1 if step < 2 else 3
        status = wk.wushkv_assign_pages(c, pool, source=torch.tensor(source, dtype=torch.int32, device=gpu))
        assert np.array_equal(status.cpu().numpy(), pages_ref.assign(h, source))
        table, refs, _ = wk.wushkv_compact_pages(c, pool, table_out=torch.empty_like(c.page_table),
                                                 refs_out=torch.empty_like(pool.refs))
        c.page_table, pool.refs = table, refs
        pages_ref.compact(h)
        for t in old:
            t.fill_(-77)
        torch.cuda.synchronize()
        assert np.array_equal(c.page_table.cpu().numpy(), h.table) and np.array_equal(pool.refs.cpu().numpy(), h.refs)
        assert np.array_equal(pool.held.cpu().numpy(), h.held) and np.array_equal(c.pages.cpu().numpy(), h.pages.reshape(-1))
