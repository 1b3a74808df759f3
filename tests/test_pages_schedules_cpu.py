"""The workgroups of the assignment's and the compaction's launches in different
orders, on the host: no result may depend on which of them a device happens to
run first."""
import copy
import types

import numpy as np
import pytest

import hostrun
import pages_ref
from hostrun import State, array
from pages_ref import Host

ORDERS = [0, 1, 5]  # ascending, descending, shuffled


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    return hostrun.build(str(tmp_path_factory.mktemp("hostrun")))


def pool_of(rng, n_pages, share, batch=3):
    """Pages of 2 560 bytes, this share of them in use, by random rows (some in
    several, some by references of the caller's own)."""
    used = rng.permutation(n_pages)[:int(n_pages * share)]
    max_pages = len(used) // batch + 7
    table = rng.choice(used, (batch, max_pages)).astype(np.int32)
    table[:, :5] = [-1, n_pages, n_pages + 3, -7, 2]
    held = np.array([max_pages, max_pages // 2, max_pages - 3][:batch], np.int32)
    refs = np.zeros(n_pages, np.int32)
    refs[used] = rng.integers(1, 5, len(used))
    pages = rng.integers(0, 256, (n_pages, 1, 2560), np.uint8)
    win = np.zeros((batch, 1, 64, 64), np.uint16)
    return types.SimpleNamespace(b=batch, hk=1, d=64, bits=2, s_sink=4, max_pages=max_pages, n_pages=n_pages, table=table,
                                 refs=refs, held=held, seq_len=np.zeros(batch), quant_end=np.zeros(batch), pages=pages,
                                 win_k=win, win_v=win)


# (a workgroup plans 4096 references)
@pytest.mark.parametrize("n_pages,share", [(3000, 0.5), (8192, 0.5), (8192, 0.05), (9000, 0.95), (20011, 0.3), (32768, 0.9),
                                           (37000, 0.6)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compaction_in_any_order(L, n_pages, share, in_place):
    rng = np.random.default_rng([n_pages, int(100 * share)])
    h = pool_of(rng, n_pages, share)
    codes = rng.integers(-128, 128, (n_pages, 1, 2, 64), np.int8)
    scales = rng.random((1, n_pages), np.float32)
    want, wcodes, wscales = copy.deepcopy(h), codes.copy(), scales.copy()
    live = pages_ref.compact(want, wcodes, wscales)
    for order in ORDERS:
        L.host_order(order)
        s, c, x = State(h), array(codes, np.int8), array(scales, np.float32)
        table, refs = (s.table, s.refs) if in_place else (array(s.table), array(s.refs))
        table_in, refs_in = s.table.copy(), s.refs.copy()
        assert s.compact(L, c, x, table, refs) == live, order
        assert np.array_equal(table, want.table) and np.array_equal(refs, want.refs), order
        assert np.array_equal(s.pages, want.pages), order
        assert np.array_equal(c, wcodes) and np.array_equal(x, wscales), order
        if not in_place:
            assert np.array_equal(s.table, table_in) and np.array_equal(s.refs, refs_in)


def same(s, h):
    return all(np.array_equal(getattr(s, n), getattr(h, n)) for n in ("table", "refs", "held", "seq_len", "quant_end", "pages",
                                                                      "win_k", "win_v"))


@pytest.mark.parametrize("seed", range(4))
def test_assignments_and_compactions_in_any_order(L, seed):
    """Random calls on a tight pool; with more than a thousand table entries
    they go through the rows in a launch of its own."""
    rng = np.random.default_rng([seed, 78])
    B = [2, 11, 40, 30][seed]
    h = Host(rng, rng.integers(0, 700, B), 1, 64, 2, spare=int(rng.integers(0, 20)), max_pages=11 if seed < 3 else 40)
    states = [State(h) for _ in ORDERS]
    for step in range(8):
        if rng.random() < 0.3:
            live = pages_ref.compact(h)
            for order, s in zip(ORDERS, states):
                L.host_order(order)
                assert s.compact(L) == live, (step, order)
        else:
            source = np.where(rng.random(B) < 0.6, np.arange(B), rng.integers(-2, B + 1, B))
            reach = rng.integers(0, 900, B) * (rng.random(B) < 0.4)
            want = pages_ref.assign(h, source, reach)
            for order, s in zip(ORDERS, states):
                L.host_order(order)
                assert np.array_equal(s.assign(L, source, reach), want), (step, order)
        for order, s in zip(ORDERS, states):
            assert same(s, h), (step, order)


def test_a_fork_copies_no_page_that_its_source_does_not_hold(L):
    """A row is valid up to held: an entry behind it, here another sequence's page,
    is not what a fork's own page is filled from."""
    h = Host(np.random.default_rng(9), [500, 333, 0], 1, 64, 2, spare=4)
    full = h.complete(0)
    assert h.every(0) == full + 1 == h.held[0]
    h.refs[h.table[0, full]] -= 1  # sequence 0 never got the page it was filling ..
    h.held[0] = full
    h.table[0, full] = h.table[1, 0]  # .. and its row names something old there
    for entries in (0, 300):  # (with many entries the rows have a launch of their own)
        big = copy.deepcopy(h)
        big.max_pages += entries
        big.table = np.pad(big.table, ((0, 0), (0, entries)), constant_values=-1)
        s = State(big)
        status = s.assign(L, [0, 1, 0])
        assert status.tolist() == [0, 0, 0] and s.held.tolist() == [full, h.held[1], full + 1]
        assert np.array_equal(s.pages, h.pages)
