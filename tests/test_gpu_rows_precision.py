"""Prefix, cross and weighted attention within a few roundings of their 64-bit
evaluation (rows_close derives how many), at every width of the codes, in states where
one source of error would stand out."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_close
import sparse_exact
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from test_gpu_rows import f32, fork, queries
from workloads import synth

pytestmark = pytest.mark.gpu


def check(what, got, want, s):
    got = got.cpu().numpy()
    assert np.isfinite(got).all()
    most, rms = rows_close.off(got, want, s)
    say("  %s: %.2e of the norm; largest %.2f, rms %.2f of what may be"
        % (what, np.linalg.norm(got - want) / np.linalg.norm(want), most, rms))
    assert most <= 1.0 and rms <= 1.0


def all_of_them(gpu, h, q, t, sel, n, leader, shared, x, source, c=None):
    c = h.cache(gpu)[0] if c is None else c
    qd, td = bf16(q, gpu), f32(t, gpu)
    for name, more in (("every page", ()), ("listed", (sel, n))):
        w = torch.zeros(h.b, h.hk, h.max_pages, device=gpu)
        got = wk.wushkv_weighted_attention(c, qd, td, w, *(dev_i32(a, gpu) for a in more))
        want, s, new, slack = rows_close.weighted(h, q, t, np.zeros(w.shape), *more)
        check(name, got, want, s)
        assert (np.abs(w.cpu().numpy().astype(np.float64) - new) <= slack).all()
    got = wk.wushkv_prefix_attention(c, qd, td, dev_i32(leader, gpu), dev_i32(shared, gpu))
    check("prefix", got, *rows_close.prefix(h, q, t, leader, shared))
    got = wk.wushkv_cross_attention(c, bf16(x, gpu), td, None, dev_i32(source, gpu))
    check("cross", got, *rows_close.cross(h, x, t, None, source))


@pytest.mark.parametrize("name", sorted(sparse_exact.STATES))
@pytest.mark.parametrize("d,bits,G,hk", [(128, 2, 4, 2), (128, 3, 4, 2), (128, 4, 8, 1), (64, 2, 8, 1), (64, 3, 1, 2), (64, 4, 2, 2),
                                         (128, 3, 1, 1)])
def test_states(gpu, name, d, bits, G, hk):
    say("%s, d %d, %d-bit, G %d" % (name, d, bits, G))
    h, q, t, sel, n = sparse_exact.state(name, d, bits, G, hk, 6, win_slots=128)
    shared = np.zeros(6, int)
    if name != "windows":
        fork(h, 2, 0, 3)
        fork(h, 1, 0, 2)
        shared[1:3] = 2, 3
    all_of_them(gpu, h, q, t, sel, n, np.array([0, 0, 0, 3, 4, 5]), shared, np.stack([q, q[::-1], q], 1), np.array([2, 1, 0, 0, 5, 1]))


@pytest.mark.parametrize("d,bits,G,hk", [(128, 2, 4, 2), (128, 3, 2, 1), (128, 4, 1, 1), (64, 3, 8, 1), (64, 4, 4, 2)])
@pytest.mark.parametrize("lens", [[1500, 900, 1200, 45, 700], [36, 4, 1, 50, 100], [3000, 40, 2000, 333, 64]])
def test_random(gpu, lens, d, bits, G, hk):
    say("%s tokens, d %d, %d-bit, G %d" % (lens, d, bits, G))
    rng = np.random.default_rng([d, bits, G, hk, lens[0]])
    h = Host(rng, lens, hk, d, bits)
    shared = np.array([0, 0, min(h.complete(0), h.complete(2)), 0, min(h.complete(2), h.complete(4))])
    fork(h, 2, 0, shared[2])
    fork(h, 4, 2, shared[4])
    q, t = queries(rng, 5, hk * G, d), pages_ref.transform(rng, hk, d)
    all_of_them(gpu, h, q, t, *sparse_exact.lists(rng, h, 9), np.array([0, 1, 0, 3, 2]), shared,
                queries(rng, 7, 5, hk * G, d), np.array([0, 4, 2, 0, 1, 3, 2]))


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("codec", ["quest", "pclip"])
def test_appended_tokens(gpu, codec, bits):
    """A cache of either codec as the append fills it."""
    say("%s, %d-bit" % (codec, bits))
    rng = np.random.default_rng([bits, len(codec)])
    lens, hk, G, d = [600, 257, 333, 3, 90], 2, 4, 128
    c = wk.WushKVCache(5, hk, d, bits, 4, 64, 8, 0.96, 0.92, max_seq_len=700, codec=codec, device=gpu)
    t = pages_ref.transform(rng, hk, d)
    k, v = (bf16(synth.to_bf16_bits(rng.standard_normal((5, 600, hk, d))), gpu) for _ in range(2))
    tk = bf16(synth.to_bf16_bits(np.stack([np.linalg.inv(x.astype(np.float64)).T for x in t])), gpu)
    wk.wushkv_append(c, k, v, dev_i32(lens, gpu), tk)
    h = object.__new__(Host)
    h.b, h.hk, h.d, h.bits, h.s_sink, h.s_keep, h.s_flush, h.win_slots = 5, hk, d, bits, 4, 64, 8, c.win_slots
    h.max_pages, h.n_pages = c.max_pages, c.n_pages
    h.table, h.seq_len, h.quant_end = (x.cpu().numpy() for x in (c.page_table, c.seq_len, c.quant_end))
    h.pages = c.pages.cpu().numpy().reshape(c.n_pages, hk, -1)
    h.win_k, h.win_v = (x.view(torch.int16).cpu().numpy().view(np.uint16) for x in (c.win_k, c.win_v))
    assert h.complete(0) >= 7
    shared = np.array([0, 3, 4, 0, 0])
    fork(h, 1, 0, shared[1])
    fork(h, 2, 0, shared[2])
    c.page_table.copy_(torch.from_numpy(h.table))
    sel, n = sparse_exact.lists(rng, h, 6)
    all_of_them(gpu, h, queries(rng, 5, hk * G, d), t, sel, n, np.array([0, 0, 0, 3, 4]), shared, queries(rng, 3, 4, hk * G, d),
                np.array([2, 0, 4]), c)
