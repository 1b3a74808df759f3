"""Weighted attention over lists that name pages several times: each entry counts, and
the weights are the same bits in every run."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_exact
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from test_gpu_rows import f32, queries

pytestmark = pytest.mark.gpu


def lists(rng, h, width, kind):
    sel = np.full((h.b, h.hk, width), -1, np.int32)
    n = np.zeros((h.b, h.hk), np.int32)
    for b in range(h.b):
        for i in range(h.hk):
            every = h.every(b)
            if kind == "random":        # any order, entries of nothing among them
                x = rng.integers(-1, every + 2, width)
            elif kind == "in turn":     # the same page far apart, in other waves and rounds
                x = np.arange(width) % max(every, 1)
            elif kind == "together":    # ascending, each several times
                x = np.sort(rng.integers(0, max(every, 1), width))
            else:                       # one page alone
                x = np.full(width, min(1, every - 1))
            sel[b, i], n[b, i] = x, rng.integers(width // 2, width + 1)
    return sel, n


@pytest.mark.parametrize("kind", ["random", "in turn", "together", "one page"])
@pytest.mark.parametrize("d,bits,G,hk,width", [(128, 2, 4, 2, 600), (64, 3, 1, 1, 257), (128, 4, 8, 1, 40), (64, 2, 2, 3, 2)])
def test_pages_listed_several_times(gpu, kind, d, bits, G, hk, width):
    say("%s, d %d, %d-bit, G %d, %d entries" % (kind, d, bits, G, width))
    rng = np.random.default_rng([d, bits, G, width, len(kind)])
    h = Host(rng, [700, 333, 120, 45, 0], hk, d, bits)
    h.table[0, 4] = -1
    q, t = queries(rng, 5, hk * G, d), pages_ref.transform(rng, hk, d)
    sel, n = lists(rng, h, width, kind)
    weights = rng.exponential(1.0, (5, hk, h.max_pages)).astype(np.float32)
    c, _ = h.cache(gpu)
    args = bf16(q, gpu), f32(t, gpu)
    runs = []
    for _ in range(20):
        w = f32(weights, gpu)
        out = wk.wushkv_weighted_attention(c, *args, w, dev_i32(sel, gpu), dev_i32(n, gpu))
        runs.append((out.cpu().numpy(), w.cpu().numpy()))
    want, s, e, new, slack = rows_exact.weighted(h, q, t, weights, sel, n)
    # rows_exact counts one sum onto what was there.  A page of k entries has k, each off
    # by u of the sum so far (all terms are positive: of the last at most): (k - 1) u more
    more = np.zeros(slack.shape)
    for b in range(5):
        for i in range(hk):
            for lp in sel[b, i, :n[b, i]]:
                if 0 <= lp < h.every(b):
                    more[b, i, lp] += 1.0
    slack += np.maximum(more - 1.0, 0.0) * rows_exact.U * new
    off, diff = rows_exact.off(runs[0][0], want, s, e), np.abs(runs[0][1].astype(np.float64) - new)
    say("  rows' errors at most %.2f of the tolerance, weights' %.2f" % (off, (diff / np.maximum(slack, 1e-300)).max()))
    assert off <= 1.0 and (diff <= slack).all()
    for out, w in runs[1:]:
        assert np.array_equal(out, runs[0][0]) and np.array_equal(w, runs[0][1])


def test_pages_far_apart(gpu):
    """Pages that differ by multiples of 4096, once and several times, and the last of a
    long row."""
    rng = np.random.default_rng(77)
    h = Host(rng, [64 * 5 + 40, 64 * 5 + 40], 2, 64, 2)
    n = 9000
    used = h.used
    h.max_pages, h.table = n, rng.choice(used, (2, n)).astype(np.int32)
    h.quant_end = np.array([4 + 64 * n - 9, 4 + 64 * 8200], np.int32)
    h.seq_len = h.quant_end + 40
    q, t = queries(rng, 2, 4, 64), pages_ref.transform(rng, 2, 64)
    sel = np.stack([np.concatenate([rng.permutation([5, 4101, 8197, 5 + 1, 4102, 8198, n - 1, n - 2, 4096, 0, 8192, 8500]),
                                    rng.integers(0, n, 288)]) for _ in range(4)]).reshape(2, 2, 300).astype(np.int32)
    sel[1, 0, 200:240] = sel[1, 0, 40]
    weights = rng.exponential(1.0, (2, 2, n)).astype(np.float32)
    c, _ = h.cache(gpu)
    runs = []
    for _ in range(5):
        w = f32(weights, gpu)
        out = wk.wushkv_weighted_attention(c, bf16(q, gpu), f32(t, gpu), w, dev_i32(sel, gpu), dev_i32(np.full((2, 2), 300), gpu))
        runs.append((out.cpu().numpy(), w.cpu().numpy()))
    want, s, e, new, slack = rows_exact.weighted(h, q, t, weights, sel, np.full((2, 2), 300))
    for b in range(2):
        for i in range(2):
            more = np.bincount(sel[b, i], minlength=n)
            slack[b, i] += np.maximum(more - 1.0, 0.0) * rows_exact.U * new[b, i]  # (as above)
    assert rows_exact.off(runs[0][0], want, s, e) <= 1.0
    assert (np.abs(runs[0][1].astype(np.float64) - new) <= slack).all()
    for out, w in runs[1:]:
        assert np.array_equal(out, runs[0][0]) and np.array_equal(w, runs[0][1])
