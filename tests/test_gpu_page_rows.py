"""Shared prefixes and eviction against their plain forms, value for value; then
both with the attentions, the assignment and the compaction, as a serving loop
runs them."""
import copy

import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_exact
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from test_gpu_rows import f32, fork, queries

pytestmark = pytest.mark.gpu


class Rows(Host):
    """Counters, page table and references alone (pages of one head of 64)."""

    def __init__(self, rng, lens, max_pages=None, spare=3, hk=1):
        super().__init__(rng, [1] * len(lens), hk, 64, 2, s_keep=32, max_pages=max_pages)
        self.seq_len = np.asarray(lens, np.int32)
        self.quant_end = np.maximum(4 + (self.seq_len - 36) // 8 * 8, 0).astype(np.int32)
        need = -(-np.maximum(self.quant_end - 4, 0) // 64)
        self.max_pages = int(max(1, need.max(), max_pages or 0))
        self.n_pages = int(need.sum()) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((self.b, self.max_pages), -1, np.int32)
        for i, end in enumerate(np.cumsum(need)):
            self.table[i, :need[i]] = order[end - need[i]:end]
        self.held = need.astype(np.int32)
        self.count()
        self.pages = np.zeros((self.n_pages, hk, self.pages.shape[2]), np.uint8)

    def count(self):
        ok = (self.table >= 0) & (self.table < self.n_pages) & (np.arange(self.max_pages) < self.held[:, None])
        self.refs = np.bincount(self.table[ok], minlength=self.n_pages).astype(np.int32)


# ------------------------------------------------------------------ prefixes


def check_prefixes(gpu, h, min_pages=1):
    c, _ = h.cache(gpu)
    leader, shared = wk.wushkv_shared_prefixes(c, min_pages=min_pages)
    torch.cuda.synchronize()
    want = pages_ref.shared_prefixes(h, min_pages)
    assert np.array_equal(leader.cpu().numpy(), want[0]) and np.array_equal(shared.cpu().numpy(), want[1])
    # (a leader leads itself)
    assert (want[0][want[0]] == want[0]).all()


@pytest.mark.parametrize("n,seed", [(1, 0), (2, 1), (9, 2), (40, 3), (70, 4)])
def test_prefixes(gpu, n, seed):
    say("prefixes of %d sequences" % n)
    rng = np.random.default_rng([n, seed])
    h = Rows(rng, rng.integers(1, 700, n), max_pages=13)
    for b in range(1, n):  # forks of earlier ones, at any depth
        if rng.random() < 0.7:
            a = int(rng.integers(0, b))
            k = int(rng.integers(0, min(h.complete(a), h.complete(b)) + 1))
            fork(h, b, a, k)
    for m in (1, 3, 100):
        check_prefixes(gpu, h, m)
    # entries that have left, in one row or in all of a group
    for b in range(n):
        gone = rng.random(13) < 0.3
        h.table[b, gone] = -1
    check_prefixes(gpu, h)
    h.table[:, 0] = -1
    check_prefixes(gpu, h)
    h.table[rng.random(h.table.shape) < 0.2] = h.n_pages  # outside the pool
    check_prefixes(gpu, h)


def test_prefixes_of_long_rows(gpu):
    rng = np.random.default_rng(7)
    lens = [64 * 600 + 50, 64 * 257 + 40, 64 * 513 + 300, 64 * 600 + 90, 64 * 256 + 40, 50]
    h = Rows(rng, lens)
    for b, a, k in ((1, 0, 257), (2, 0, 512), (3, 0, 599), (4, 2, 255)):
        fork(h, b, a, k)
    check_prefixes(gpu, h)
    h.table[[0, 3], 300:] = -1
    check_prefixes(gpu, h)


def test_prefixes_of_a_large_batch(gpu):
    """More sequences than one sweep of the workgroup takes."""
    rng = np.random.default_rng(8)
    n = 1100
    h = Rows(rng, rng.integers(100, 300, n))
    lead = rng.integers(0, 7, n)
    for b in range(7, n):
        fork(h, b, int(lead[b]), min(int(rng.integers(0, 4)), h.complete(b), h.complete(int(lead[b]))))
    check_prefixes(gpu, h)


# ------------------------------------------------------------------ eviction


def check_evict(gpu, h, weights, budget, recent, max_sel, in_place):
    c, pool = h.cache(gpu)
    pool.low.fill_(0)
    sel = torch.full((h.b, h.hk, max_sel), 77, dtype=torch.int32, device=gpu)
    n_sel, gone = dev_i32(np.full((h.b, h.hk), 99), gpu), dev_i32(np.full(h.b, 99), gpu)
    table, refs = c.page_table.clone(), pool.refs.clone()
    other = {} if in_place else dict(table_out=torch.full_like(table, 55), refs_out=torch.full_like(refs, 55))
    wk.wushkv_evict_pages(c, pool, f32(weights, gpu), dev_i32(budget, gpu), recent=recent, sel=sel, n_sel=n_sel, evicted=gone,
                          **other)
    torch.cuda.synchronize()
    new = [x.cpu().numpy() for x in (other.get("table_out", c.page_table), other.get("refs_out", pool.refs), sel, n_sel, gone)]
    if other:
        assert torch.equal(c.page_table, table) and torch.equal(pool.refs, refs)
    h = copy.deepcopy(h)
    want = pages_ref.evict(h, weights, budget, recent, max_sel)
    for got, x in zip(new, (h.table, h.refs, *want)):
        assert np.array_equal(got, x)
    assert pool.low.item() == 0
    return h


@pytest.mark.parametrize("hk,seed", [(1, 0), (3, 1), (8, 2)])
def test_evict(gpu, hk, seed):
    say("evict, %d heads" % hk)
    rng = np.random.default_rng([hk, seed])
    h = Rows(rng, [1, 36, 100, 101, 333, 700, 700, 64 * 12 + 36 + 4, 500, 0], max_pages=14, hk=hk)
    fork(h, 6, 5, 9)
    fork(h, 8, 5, 4)
    h.table[5, 3] = h.table[7, 0] = -1
    h.table[4, 1] = h.n_pages + 2
    h.held[8] = 6  # (its row is not read behind that)
    h.count()
    # few values, so that ties are many; weights that are not numbers, negative, infinite
    w = rng.integers(-1, 3, (h.b, hk, 14)).astype(np.float32)
    w[5, 0, :3] = [np.nan, np.inf, -np.inf]
    for budget, recent, max_sel in ((0, 0, 14), (3, 0, 14), (3, 2, 5), (5, 20, 14), (100, 0, 2), (2, 1, 1)):
        each = np.full(h.b, budget)
        each[9] = -1
        each[6] = budget - 1
        for in_place in (False, True):
            check_evict(gpu, h, w, each, recent, max_sel, in_place)
    check_evict(gpu, h, rng.standard_normal(w.shape).astype(np.float32), np.full(h.b, 4), 1, 20, True)


def test_evict_long_rows(gpu):
    """Rows of several sweeps, and one whose keys do not stay in LDS."""
    rng = np.random.default_rng(5)
    h = Rows(rng, [64 * 9000 + 77, 64 * 1500 + 90, 64 * 8192 + 36 + 4], hk=2)
    h.table[rng.random(h.table.shape) < 0.1] = -1
    h.count()
    w = (rng.integers(0, 40, (3, 2, h.max_pages)) * 0.25).astype(np.float32)
    for budget, recent in ((4000, 10), (100, 0), (0, 3)):
        check_evict(gpu, h, w, np.full(3, budget), recent, h.max_pages, True)


def test_evict_without_lists(gpu):
    rng = np.random.default_rng(6)
    h = Rows(rng, [700, 500])
    c, pool = h.cache(gpu)
    w, budget = f32(rng.exponential(1.0, (2, 1, h.max_pages)), gpu), dev_i32([2, 3], gpu)
    pool.low.fill_(h.n_pages)
    sel, n_sel, gone = wk.wushkv_evict_pages(c, pool, w, budget, max_sel=0)
    torch.cuda.synchronize()
    assert sel.shape == (2, 1, 0)
    pages_ref.evict(h, w.cpu().numpy(), [2, 3], 0, 1)
    assert np.array_equal(c.page_table.cpu().numpy(), h.table) and np.array_equal(pool.refs.cpu().numpy(), h.refs)
    # the lowest page that became free
    before = Rows(np.random.default_rng(6), [700, 500])
    assert pool.low.item() == min(np.flatnonzero((before.refs > 0) & (h.refs == 0)))
