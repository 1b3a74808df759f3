"""Refusals and sizes of the page operators and the sparse attention, which
need no GPU, and the tests' own plain forms against brute force."""
import ctypes

import numpy as np
import pytest
import torch

import pages_ref
from conftest import gpu_available
from test_abi_cpu import FAKE, _desc

wk = pytest.importorskip("paper_2609_38121_amd")
from paper_2609_38121_amd import _lib  # noqa: E402

no_gpu = pytest.mark.skipif(gpu_available(), reason="fake device pointers: run only where no GPU exists")
BIG = 1 << 40


def refs(**over):
    c = _lib.CacheDesc.from_buffer_copy(_desc(**over))
    return ctypes.byref(c), ctypes.byref(_lib.BoundsDesc(FAKE, FAKE)), ctypes.byref(_lib.PoolDesc(FAKE, FAKE, FAKE))


def calls(L, c, b, p):
    """Every entry point with its good arguments: name -> (function, arguments)."""
    return {
        "bounds": (L.wushkv_page_bounds, [c, b, FAKE, 4, None]),
        "select": (L.wushkv_select_pages, [c, b, FAKE, 8, 200, FAKE, 2, FAKE, FAKE, FAKE, FAKE, BIG, None]),
        "sparse": (L.wushkv_sparse_attention, [c, FAKE, 8, FAKE, FAKE, 3, FAKE, 0.1, FAKE, FAKE, BIG, None]),
        "assign": (L.wushkv_assign_pages, [c, p, FAKE, FAKE, FAKE, None]),
        "compact": (L.wushkv_compact_pages, [c, p, b, FAKE, FAKE, FAKE, FAKE, BIG, None]),
    }


@no_gpu
@pytest.mark.parametrize("over,status", [(dict(batch=0), -1), (dict(head_dim=96), -2), (dict(bits=5), -2),
                                         (dict(seq_len=None), -1), (dict(pages=None), -1), (dict(codec=7), -1)])
def test_bad_caches_are_refused(over, status):
    L = _lib.lib()
    c, b, p = refs(**over)
    for name, (f, args) in calls(L, c, b, p).items():
        assert f(*args) == status, name
        assert f(None, *args[1:]) == -1, name
    assert L.wushkv_select_workspace_bytes(c, 8, 200, 2) == 0
    assert L.wushkv_sparse_workspace_bytes(c, 8, 3) == 0
    assert L.wushkv_compact_workspace_bytes(c) == 0


BAD = [  # entry point, argument, value, status
    ("bounds", 1, None, -1), ("bounds", 2, FAKE + 4, -1), ("bounds", 3, -1, -1), ("bounds", 3, 0, 0),
    ("select", 1, None, -1), ("select", 2, None, -1), ("select", 2, FAKE + 2, -1), ("select", 3, 7, -1),
    ("select", 3, 0, -1), ("select", 3, 6, -2), ("select", 3, 32, -2), ("select", 4, -1, -1), ("select", 5, None, -1),
    ("select", 5, FAKE + 4, -1), ("select", 6, -1, -1), ("select", 6, 2 ** 31 - 1, -1), ("select", 7, None, -1),
    ("select", 8, None, -1), ("select", 8, FAKE + 4, -1), ("select", 9, FAKE + 4, -1), ("select", 10, None, -1),
    ("select", 11, 16, -3),
    ("sparse", 1, None, -1), ("sparse", 2, 7, -1), ("sparse", 2, 32, -2), ("sparse", 3, None, -1),
    ("sparse", 3, FAKE + 4, -1), ("sparse", 4, None, -1), ("sparse", 5, -1, -1), ("sparse", 5, 300000, -2),
    ("sparse", 6, None, -1), ("sparse", 7, 0.0, -1), ("sparse", 7, float("nan"), -1), ("sparse", 7, float("inf"), -1),
    ("sparse", 8, None, -1), ("sparse", 9, None, -1), ("sparse", 10, 16, -3),
    ("assign", 1, None, -1), ("assign", 2, FAKE + 4, -1), ("assign", 3, FAKE + 4, -1), ("assign", 4, None, -1),
    ("assign", 4, FAKE + 4, -1),
    ("compact", 1, None, -1), ("compact", 3, None, -1), ("compact", 4, None, -1), ("compact", 4, FAKE + 4, -1),
    ("compact", 5, FAKE + 4, -1), ("compact", 6, None, -1), ("compact", 7, 16, -3),
]


@no_gpu
@pytest.mark.parametrize("name,at,value,status", BAD)
def test_bad_arguments_are_refused(name, at, value, status):
    L = _lib.lib()
    f, args = calls(L, *refs())[name]
    args[at] = value
    assert f(*args) == status


@no_gpu
def test_bad_boxes_and_pools_are_refused():
    L = _lib.lib()
    c, b, p = refs()
    for bad in (_lib.BoundsDesc(None, FAKE), _lib.BoundsDesc(FAKE, None), _lib.BoundsDesc(FAKE + 4, FAKE)):
        got = calls(L, c, ctypes.byref(bad), p)
        assert [got[n][0](*got[n][1]) for n in ("bounds", "select", "compact")] == [-1] * 3
    for bad in (_lib.PoolDesc(None, FAKE, FAKE), _lib.PoolDesc(FAKE, None, FAKE), _lib.PoolDesc(FAKE, FAKE, None),
                _lib.PoolDesc(FAKE, FAKE + 4, FAKE)):
        got = calls(L, c, b, ctypes.byref(bad))
        assert [got[n][0](*got[n][1]) for n in ("assign", "compact")] == [-1] * 2
    # batches and tables beyond what the plans number
    f, args = calls(L, *refs(batch=16385))["assign"]
    assert f(*args) == -2
    f, args = calls(L, *refs(batch=16384, max_pages_per_seq=1 << 18))["assign"]
    assert f(*args) == -2
    # a cache without pages has nothing to move
    f, args = calls(L, *refs(n_pages=0))["compact"]
    assert f(*args) == -1


def test_workspace_sizes():
    L = _lib.lib()
    c = ctypes.byref(_desc())
    # a plan over a list has the sizes of one over as many pages
    for pages in (0, 1, 4, 16):
        assert L.wushkv_sparse_workspace_bytes(c, 8, pages) == L.wushkv_decode_workspace_bytes(c, 8, 4 + 64 * pages)
    # at least a score per page of every (sequence, kv head)
    assert L.wushkv_select_workspace_bytes(c, 8, 200, 2) >= 2 * 2 * 4 * 4
    assert L.wushkv_compact_workspace_bytes(c) >= 4 * 8


def test_bindings_check_tensors():
    c = wk.WushKVCache(2, 2, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=200, device="cpu", page_order="none", n_pages=5)
    assert c.n_pages == 5 and (c.page_table == -1).all()
    with pytest.raises(ValueError):
        wk.WushKVCache(2, 2, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=200, device="cpu", n_pages=5)
    pool, bounds = wk.WushKVPool(c), wk.WushKVBounds(c)
    assert pool.refs.tolist() == [0] * 5 and pool.held.tolist() == [0, 0]
    full = wk.WushKVCache(2, 2, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=200, device="cpu", page_order="random",
                          pool_factor=2.0)
    counts = wk.WushKVPool(full)
    assert counts.refs.sum() == 2 * full.max_pages and counts.held.tolist() == [full.max_pages] * 2
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, t = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 64, 64)
    bad = [
        lambda: wk.wushkv_page_bounds(c, bounds, since=i32(3)),
        lambda: wk.wushkv_page_bounds(c, bounds, since=i32(2).long()),
        lambda: wk.wushkv_select_pages(c, bounds, q.float(), t, 2),
        lambda: wk.wushkv_select_pages(c, bounds, q[:1], t, 2),
        lambda: wk.wushkv_select_pages(c, bounds, q, t.transpose(1, 2), 2),
        lambda: wk.wushkv_select_pages(c, bounds, q, t, 2, scores=torch.zeros(2, 2, 1)),
        lambda: wk.wushkv_sparse_attention(c, q, t, i32(2, 2), i32(2, 2)),
        lambda: wk.wushkv_sparse_attention(c, q, t, i32(2, 2, 3)[:, :, ::2], i32(2, 2)),
        lambda: wk.wushkv_sparse_attention(c, q, t, i32(2, 2, 3), i32(2)),
        lambda: wk.wushkv_page_bounds(c, wk.WushKVBounds(full)),
        lambda: wk.wushkv_select_pages(c, wk.WushKVBounds(full), q, t, 2),
        lambda: wk.wushkv_select_pages(c, bounds, q, t, 2, workspace=i32(8, 8)[:, ::2]),
        lambda: wk.wushkv_sparse_attention(c, q, t, i32(2, 2, 3), i32(2, 2), workspace=i32(8, 8)[:, ::2]),
        lambda: wk.wushkv_assign_pages(c, counts),
        lambda: wk.wushkv_compact_pages(c, counts),
        lambda: wk.wushkv_compact_pages(c, pool, bounds=wk.WushKVBounds(full)),
        lambda: wk.wushkv_assign_pages(c, pool, source=i32(1)),
        lambda: wk.wushkv_assign_pages(c, pool, reach=i32(2).float()),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_plain_box_holds_its_keys():
    rng = np.random.default_rng(3)
    h = pages_ref.Host(rng, [300], 2, 64, 2)
    for p in h.used:
        for k in range(2):
            x = h.stored(p, k)
            c, s = pages_ref.box(x)
            c = c.astype(np.float64)
            slack = 2.0 ** -20 * np.abs(x).max()
            assert (x <= (c[0] + c[1]) * s + slack).all() and (x >= (c[0] - c[1]) * s - slack).all()
            assert (c[1] * s <= (x.max(0) - x.min(0)) / 2 + 1.51 * s).all()


def test_plain_scores_bound_the_logits():
    rng = np.random.default_rng(4)
    h = pages_ref.Host(rng, [500, 90], 2, 64, 4)
    t = pages_ref.transform(rng, 2, 64)
    q = pages_ref.synth.to_bf16_bits(rng.standard_normal((2, 4, 64)))
    codes, scales = np.zeros((h.n_pages, 2, 2, 64), np.int8), np.zeros((2, h.n_pages), np.float32)
    for p in h.used:
        for k in range(2):
            codes[p, k], scales[k, p] = pages_ref.box(h.stored(p, k))
    score = pages_ref.scores(h, codes, scales, q, t)
    x = pages_ref.synth.bf16_bits_to_float(q).astype(np.float64)
    for b in range(2):
        for k in range(2):
            qt = x[b, 2 * k:2 * k + 2] @ t[k].astype(np.float64)
            for lp in range(h.complete(b)):
                keys = h.stored(h.table[b, lp], k)
                most = (qt @ keys.T).max()
                # N is off by half a unit of 2^-F <= 2^-13 max |q~| an entry
                slack = 2.0 ** -14 * np.abs(qt).max() * np.abs(keys).sum(1).max() * 1.1
                assert most <= score[b, k, lp] + slack
    sel, n = pages_ref.select(h, score, 2)
    assert n[0, 0] == 2 + (h.every(0) > h.complete(0)) and (np.diff(sel[0, 0, :n[0, 0]]) > 0).all()
