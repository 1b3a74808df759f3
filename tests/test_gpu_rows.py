"""Attention of many query rows over stored sequences: shared prefixes, cross
attention, and attention that adds up the pages' weights, against the definitions
in 64 bits (tests/rows_exact.py)."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_exact
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from workloads import synth

pytestmark = pytest.mark.gpu

SHAPES = [(64, 2, 1, 2), (64, 4, 4, 1), (64, 2, 8, 1), (64, 3, 2, 3), (128, 2, 4, 2), (128, 4, 8, 1), (128, 4, 1, 5),
          (128, 2, 8, 2), (128, 3, 2, 1), (128, 2, 1, 1)]


def queries(rng, *shape):
    return synth.to_bf16_bits(rng.standard_normal(shape))


def f32(a, gpu):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(gpu)


def fork(h, b, src, pages):
    """Sequence b's first pages become src's."""
    h.table[b, :pages] = h.table[src, :pages]


def dirty(h):
    """NaN patterns in dead window slots and behind the quantised positions."""
    for b in range(h.b):
        S, end = int(h.seq_len[b]), h.end(b)
        ring = h.win_slots - h.s_sink
        live = [p if p < h.s_sink else h.s_sink + (p - h.s_sink) % ring for p in range(S) if p < h.s_sink or p >= end]
        dead = np.setdiff1d(np.arange(h.win_slots), live)
        h.win_k[b][:, dead] = 0x7FC1
        h.win_v[b][:, :, dead] = 0xFFFF
        if h.every(b) > h.complete(b):
            first = end - h.s_sink - 64 * h.complete(b)
            par = h.pages.shape[2] - 512
            page = h.pages[h.table[b, h.complete(b)]]
            page[:, par + 4 * first:par + 256] = 0xFF
            page[:, par + 256 + 4 * first:] = 0xFF


# ------------------------------------------------------------------ prefixes


def run_prefix(gpu, h, q, t, leader, shared, **kw):
    c, _ = h.cache(gpu)
    out = torch.full((h.b, q.shape[1], h.d), float("nan"), device=gpu)
    wk.wushkv_prefix_attention(c, bf16(q, gpu), f32(t, gpu), dev_i32(leader, gpu), dev_i32(shared, gpu), out=out, **kw)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    want, s, w = rows_exact.prefix(h, q, t, leader, shared)
    off = rows_exact.off(got, want, s, w)
    say("  rows' errors at most %.2f of the tolerance" % off)
    assert off <= 1.0
    return got


@pytest.mark.parametrize("d,bits,G,hk", SHAPES)
def test_prefix(gpu, d, bits, G, hk):
    say("prefix d %d, %d-bit, G %d, %d heads" % (d, bits, G, hk))
    rng = np.random.default_rng([d, bits, G, hk, 1])
    # a group of six of different depth, one of two, alone, empty, one token
    h = Host(rng, [700, 333, 650, 0, 500, 640, 36 + 4 + 320, 1, 420, 600], hk, d, bits)
    for b, src, n in ((2, 0, 7), (4, 0, 3), (5, 0, 8), (6, 0, 4), (9, 0, 7), (8, 1, 2)):
        fork(h, b, src, n)
    dirty(h)
    leader = np.arange(10)
    shared = np.zeros(10, int)
    for b, src, n in ((2, 0, 7), (4, 0, 3), (5, 0, 8), (6, 0, 4), (9, 0, 7), (8, 1, 2)):
        leader[b], shared[b] = src, n
    q, t = queries(rng, 10, hk * G, d), pages_ref.transform(rng, hk, d)
    got = run_prefix(gpu, h, q, t, leader, shared)
    assert (got[3] == 0).all()
    # nothing shared, as a plain decode
    run_prefix(gpu, h, q, t, np.arange(10), np.zeros(10, int))
    # leaders outside the batch, counts beyond what there is, a leader that follows
    # another, other sequences' pages
    run_prefix(gpu, h, q, t, np.array([-1, 0, 1, 2, 10, 4, 5, 0, 2, 1 << 30]), np.array([5, 99, 2, 3, 4, -2, 1 << 30, 5, 1, 7]))
    # pages that have left the row
    h.table[0, 1] = h.table[5, 1] = -1
    h.table[1, 1] = h.n_pages
    run_prefix(gpu, h, q, t, leader, shared)


@pytest.mark.parametrize("d,bits,G,hk,n", [(128, 2, 4, 8, 40), (128, 4, 8, 2, 70), (64, 2, 1, 3, 130)])
def test_prefix_of_many(gpu, d, bits, G, hk, n):
    """Several tiles of one group, and workgroups that take parts of tiles."""
    say("prefix of %d sequences, d %d, %d-bit, G %d, %d heads" % (n, d, bits, G, hk))
    rng = np.random.default_rng([n, d])
    lens = rng.integers(3 * 64 + 40, 20 * 64, n)
    lens[0] = 24 * 64
    h = Host(rng, lens, hk, d, bits, win_slots=128, s_keep=50)
    shared = np.array([0] + [int(rng.integers(1, h.complete(b) + 1)) for b in range(1, n)])
    for b in range(1, n):
        fork(h, b, 0, shared[b])
    leader = np.zeros(n, int)
    run_prefix(gpu, h, queries(rng, n, hk * G, d), pages_ref.transform(rng, hk, d), leader, shared)


# ------------------------------------------------------------------ cross


def run_cross(gpu, h, q, t, n_tok=None, source=None, **kw):
    c, _ = h.cache(gpu)
    out = torch.full(q.shape, float("nan"), device=gpu)
    wk.wushkv_cross_attention(c, bf16(q, gpu), f32(t, gpu), None if n_tok is None else dev_i32(n_tok, gpu),
                              None if source is None else dev_i32(source, gpu), out=out, **kw)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    want, s, w = rows_exact.cross(h, q, t, n_tok, source)
    off = rows_exact.off(got, want, s, w)
    say("  rows' errors at most %.2f of the tolerance" % off)
    assert off <= 1.0
    return got


@pytest.mark.parametrize("d,bits,G,hk", SHAPES)
def test_cross(gpu, d, bits, G, hk):
    say("cross d %d, %d-bit, G %d, %d heads" % (d, bits, G, hk))
    rng = np.random.default_rng([d, bits, G, hk, 2])
    h = Host(rng, [0, 1, 4, 36, 45, 100, 333, 700], hk, d, bits)
    dirty(h)
    t = pages_ref.transform(rng, hk, d)
    # one token of each; several, in any order, of outside and of nothing
    run_cross(gpu, h, queries(rng, 8, 1, hk * G, d), t)
    source = np.array([7, 6, 0, 7, -1, 5, 8, 7, 1, 6, 4, 7])
    n_tok = np.array([5, 1, 3, 0, 2, 9, 4, 7, -3, 6, 2, 1])
    got = run_cross(gpu, h, queries(rng, 12, 7, hk * G, d), t, n_tok, source)
    assert (got[2] == 0).all() and (got[4] == 0).all() and (got[0, 5:] == 0).all()


@pytest.mark.parametrize("d,bits,G,hk,tok,lens", [(128, 2, 4, 2, 37, [900, 70]), (64, 2, 1, 1, 300, [260]), (128, 4, 8, 1, 9, [3000])])
def test_cross_of_many_tokens(gpu, d, bits, G, hk, tok, lens):
    say("cross, %d tokens over %s, d %d, %d-bit, G %d" % (tok, lens, d, bits, G))
    rng = np.random.default_rng([tok, d])
    h = Host(rng, lens, hk, d, bits, win_slots=192, s_keep=150)
    run_cross(gpu, h, queries(rng, len(lens), tok, hk * G, d), pages_ref.transform(rng, hk, d))


# ------------------------------------------------------------------ weighted


def run_weighted(gpu, h, q, t, weights, sel=None, n_sel=None, **kw):
    c, _ = h.cache(gpu)
    out = torch.full((h.b, q.shape[1], h.d), float("nan"), device=gpu)
    w = f32(weights, gpu)
    wk.wushkv_weighted_attention(c, bf16(q, gpu), f32(t, gpu), w, None if sel is None else dev_i32(sel, gpu),
                                 None if sel is None else dev_i32(n_sel, gpu), out=out, **kw)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    want, s, e, new, slack = rows_exact.weighted(h, q, t, weights, sel, n_sel)
    off = rows_exact.off(got, want, s, e)
    diff = np.abs(w.cpu().numpy().astype(np.float64) - new)
    say("  rows' errors at most %.2f of the tolerance, weights' %.2f" % (off, (diff / np.maximum(slack, 1e-300)).max()))
    assert off <= 1.0 and (diff <= slack).all()
    return got, w.cpu().numpy()


@pytest.mark.parametrize("d,bits,G,hk", SHAPES)
def test_weighted(gpu, d, bits, G, hk):
    say("weighted d %d, %d-bit, G %d, %d heads" % (d, bits, G, hk))
    rng = np.random.default_rng([d, bits, G, hk, 3])
    h = Host(rng, [0, 1, 4, 36, 45, 100, 333, 700], hk, d, bits, max_pages=13)
    dirty(h)
    q, t = queries(rng, 8, hk * G, d), pages_ref.transform(rng, hk, d)
    weights = rng.exponential(1.0, (8, hk, 13)).astype(np.float32)
    got, w = run_weighted(gpu, h, q, t, weights)
    assert (got[0] == 0).all() and np.array_equal(w[0], weights[0])
    assert np.array_equal(w[7, :, h.every(7):], weights[7, :, h.every(7):])
    # pages that have left; lists in any order, with entries of nothing
    h.table[7, 2], h.table[6, 0] = -1, h.n_pages
    run_weighted(gpu, h, q, t, np.zeros_like(weights))
    sel = rng.permuted(np.broadcast_to(np.arange(-1, 14), (8, hk, 15)), axis=2)
    n_sel = rng.integers(-1, 17, (8, hk))
    run_weighted(gpu, h, q, t, weights, sel, n_sel)
    run_weighted(gpu, h, q, t, weights, np.zeros((8, hk, 0)), np.ones((8, hk)))
