"""Refusals of the attentions of many query rows, of shared prefixes and of
eviction, before anything is enqueued."""
import ctypes

import pytest

from conftest import gpu_available
from test_abi_cpu import BAD, FAKE, _desc

wk = pytest.importorskip("paper_2609_38121_amd")
from paper_2609_38121_amd import _lib  # noqa: E402

pytestmark = pytest.mark.skipif(gpu_available(), reason="fake device pointers: run only where no GPU exists")

P, ODD = FAKE, FAKE + 4
BIG = 1 << 40


def prefixes(c, min_pages=1, leader=P, shared=P):
    return _lib.lib().wushkv_shared_prefixes(ctypes.byref(c), min_pages, leader, shared, None)


def prefix(c, q=P, n_q=4, leader=P, shared=P, t=P, scale=0.1, out=P, ws=P, n=BIG):
    return _lib.lib().wushkv_prefix_attention(ctypes.byref(c), q, n_q, leader, shared, t, scale, out, ws, n, None)


def cross(c, q=P, n=2, n_tok=P, tok=3, source=P, n_q=4, t=P, scale=0.1, out=P, ws=P, size=BIG):
    return _lib.lib().wushkv_cross_attention(ctypes.byref(c), q, n, n_tok, tok, source, n_q, t, scale, out, ws, size, None)


def weighted(c, q=P, n_q=4, sel=P, n_sel=P, width=3, t=P, scale=0.1, w=P, out=P, ws=P, n=BIG):
    return _lib.lib().wushkv_weighted_attention(ctypes.byref(c), q, n_q, sel, n_sel, width, t, scale, w, out, ws, n, None)


def evict(c, refs=P, held=P, low=P, w=P, budget=P, recent=0, table=P, refs_out=P, sel=P, n_sel=P, width=3, gone=P, pool=True):
    books = ctypes.byref(_lib.PoolDesc(refs, held, low)) if pool else None
    return _lib.lib().wushkv_evict_pages(ctypes.byref(c), books, w, budget, recent, table, refs_out, sel, n_sel, width, gone, None)


@pytest.mark.parametrize("over,status", BAD)
@pytest.mark.parametrize("call", [prefixes, prefix, cross, weighted, evict])
def test_descriptors(call, over, status):
    assert call(_desc(**over)) == status


@pytest.mark.parametrize("call", [prefix, cross, weighted])
def test_attentions(call):
    c = _desc()
    assert call(c, n_q=3) == -1 and call(c, n_q=0) == -1
    assert call(c, n_q=6) == -2 and call(c, n_q=32) == -2
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call(c, scale=scale) == -1
    for name in ("q", "t", "out", "ws"):
        assert call(c, **{name: None}) == -1 and call(c, **{name: ODD}) == -1


def test_sizes():
    c = _desc()
    for name in ("leader", "shared"):
        assert prefixes(c, **{name: None}) == -1 and prefixes(c, **{name: ODD}) == -1
        assert prefix(c, **{name: None}) == -1 and prefix(c, **{name: ODD}) == -1
    assert prefixes(c, min_pages=0) == -1
    assert prefix(_desc(batch=1025)) == -2
    assert cross(c, n=0) == -1 and cross(c, tok=0) == -1 and cross(c, source=None, n=3) == -1
    assert cross(c, n=1025) == -2 and cross(c, n=2, tok=131073) == -2
    assert cross(c, n_tok=ODD) == -1 and cross(c, source=ODD) == -1
    assert weighted(c, w=None) == -1 and weighted(c, w=ODD) == -1 and weighted(c, sel=ODD) == -1 and weighted(c, n_sel=ODD) == -1
    # half a list
    assert weighted(c, sel=None) == -1 and weighted(c, n_sel=None) == -1 and weighted(c, width=-2) == -1
    assert weighted(c, sel=None, n_sel=None) == -1 and weighted(c, width=-1) == -1
    assert weighted(_desc(batch=65536)) == -2


def test_workspaces():
    c, L = _desc(), _lib.lib()
    need = [L.wushkv_prefix_workspace_bytes(ctypes.byref(c), 4), L.wushkv_cross_workspace_bytes(ctypes.byref(c), 2, 3, 4),
            L.wushkv_weighted_workspace_bytes(ctypes.byref(c), 4, 3)]
    assert all(n > 0 for n in need)
    assert prefix(c, n=need[0] - 1) == -3 and cross(c, size=need[1] - 1) == -3 and weighted(c, n=need[2] - 1) == -3
    assert L.wushkv_weighted_workspace_bytes(ctypes.byref(c), 4, -1) > 0
    assert L.wushkv_prefix_workspace_bytes(ctypes.byref(c), 3) == 0
    assert L.wushkv_prefix_workspace_bytes(ctypes.byref(_desc(batch=1025)), 4) == 0
    assert L.wushkv_cross_workspace_bytes(ctypes.byref(c), 0, 3, 4) == 0
    assert L.wushkv_cross_workspace_bytes(ctypes.byref(c), 2, 131073, 4) == 0
    assert L.wushkv_weighted_workspace_bytes(ctypes.byref(_desc(batch=0)), 4, 3) == 0


def test_evictions():
    c = _desc()
    assert evict(c, pool=False) == -1 and evict(c, recent=-1) == -1 and evict(c, width=-1) == -1
    for name in ("refs", "held", "low", "w", "budget", "table", "refs_out", "gone"):
        assert evict(c, **{name: None}) == -1 and evict(c, **{name: ODD}) == -1
    assert evict(c, sel=None) == -1 and evict(c, n_sel=None) == -1 and evict(c, sel=ODD) == -1 and evict(c, n_sel=ODD) == -1
