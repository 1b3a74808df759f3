"""Plans of many tiles: batches, query sequences and tokens up to the largest that the
calls take, with tiles of every size, so that a plan's workgroup goes over its tiles,
items and sorted sequences several times.

A few stored sequences and query rows are evaluated in 64 bits; a batch repeats them
in any order, and every row of it is checked."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_close
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from test_gpu_rows import f32, queries

pytestmark = pytest.mark.gpu

# nothing, a token, windows alone, the page being filled, a few pages, long ones
LENS = [0, 1, 20, 36, 50, 101, 110, 170, 240, 333, 700, 1500]


def repeated(h, idx, gpu):
    """The cache whose sequence i is h's sequence idx[i] (its pages too)."""
    one, _ = h.cache(gpu)
    c = wk.WushKVCache(len(idx), h.hk, h.d, h.bits, h.s_sink, h.s_keep, h.s_flush, 0.96, 0.92,
                       max_seq_len=h.s_sink + 64 * h.max_pages, win_slots=h.win_slots, page_order="none", n_pages=h.n_pages,
                       device=gpu)
    c.pages.copy_(one.pages)
    at = torch.from_numpy(idx).to(gpu)
    for name in ("page_table", "win_k", "win_v", "seq_len", "quant_end"):
        getattr(c, name).copy_(getattr(one, name)[at])
    return c


def check(got, want, s):
    """Every repetition's rows within their roundings (rows of no tokens are zeros)."""
    e = np.linalg.norm(got.astype(np.float64) - want, axis=-1)
    say("  rows' errors at most %.2f of what may be" % (e[s > 0] / (3.0 * s[s > 0])).max())
    assert (e <= 3.0 * s).all()


@pytest.mark.parametrize("d,bits,G,hk,n", [(64, 2, 2, 2, 700), (128, 4, 8, 1, 1100), (128, 2, 1, 3, 2500), (64, 3, 1, 1, 65535)])
def test_weighted_batches(gpu, d, bits, G, hk, n):
    say("weighted, %d sequences, d %d, %d-bit, G %d" % (n, d, bits, G))
    rng = np.random.default_rng([n, d])
    h = Host(rng, LENS, hk, d, bits)
    q, t = queries(rng, len(LENS), hk * G, d), pages_ref.transform(rng, hk, d)
    want, s, new, slack = rows_close.weighted(h, q, t, np.zeros((len(LENS), hk, h.max_pages)))
    # (the long ones are few: what is cut lies among what is not)
    idx = rng.choice(len(LENS), n, p=np.array([10.0] * 10 + [1.0, 1.0]) / 102.0)
    c = repeated(h, idx, gpu)
    weights = torch.zeros(n, hk, h.max_pages, device=gpu)
    out = wk.wushkv_weighted_attention(c, bf16(q[idx], gpu), f32(t, gpu), weights)
    check(out.cpu().numpy(), want[idx], s[idx])
    assert (np.abs(weights.cpu().numpy() - new[idx]) <= slack[idx]).all()


@pytest.mark.parametrize("d,bits,G,hk,n", [(64, 2, 8, 1, 1024), (128, 3, 1, 2, 1024), (128, 4, 4, 1, 900), (64, 4, 1, 2, 600)])
def test_prefix_batches(gpu, d, bits, G, hk, n):
    say("prefix, %d sequences, d %d, %d-bit, G %d" % (n, d, bits, G))
    rng = np.random.default_rng([n, d, 2])
    h = Host(rng, LENS, hk, d, bits)
    few = queries(rng, 3, len(LENS), hk * G, d)
    t = pages_ref.transform(rng, hk, d)
    alone = np.arange(len(LENS)), np.zeros(len(LENS), int)
    each = [rows_close.prefix(h, x, t, *alone) for x in few]
    want, s = (np.stack([e[i] for e in each]) for i in (0, 1))
    idx, which = rng.integers(0, len(LENS), n), rng.integers(0, 3, n)
    c, q = repeated(h, idx, gpu), bf16(few[which, idx], gpu)
    leader, shared = wk.wushkv_shared_prefixes(c)
    full = np.array([h.complete(b) for b in idx])
    first = np.array([np.flatnonzero(idx == b)[0] for b in idx])
    assert np.array_equal(leader.cpu().numpy(), np.where(full > 0, first, np.arange(n)))
    assert np.array_equal(shared.cpu().numpy(), np.where(first == np.arange(n), 0, full))
    out = wk.wushkv_prefix_attention(c, q, f32(t, gpu), leader, shared)
    check(out.cpu().numpy(), want[which, idx], s[which, idx])
    # any leader with the same pages, any part of them
    some = np.array([rng.choice(np.flatnonzero(idx == b)) for b in idx])
    out = wk.wushkv_prefix_attention(c, q, f32(t, gpu), dev_i32(some, gpu), dev_i32(rng.integers(0, 30, n), gpu))
    check(out.cpu().numpy(), want[which, idx], s[which, idx])


@pytest.mark.parametrize("d,bits,G,hk,n,tok", [(64, 2, 1, 2, 1024, 3), (128, 3, 4, 1, 300, 40), (128, 2, 8, 2, 70, 9),
                                               (64, 4, 2, 1, 5, 2000), (64, 2, 8, 1, 1024, 128)])
def test_cross_batches(gpu, d, bits, G, hk, n, tok):
    say("cross, %d sequences of %d tokens, d %d, %d-bit, G %d" % (n, tok, d, bits, G))
    rng = np.random.default_rng([n, tok, d, 3])
    h = Host(rng, LENS, hk, d, bits)
    t = pages_ref.transform(rng, hk, d)
    # seven tokens, over every stored sequence (a source outside the batch: zeros)
    few = queries(rng, 7, hk * G, d)
    want, s = rows_close.cross(h, np.broadcast_to(few, (13, *few.shape)), t, None, np.array([*range(12), -1]))
    source, which = rng.integers(0, 13, n), rng.integers(0, 7, (n, tok))
    n_tok = np.where(rng.random(n) < 0.5, tok, rng.integers(0, tok + 1, n))
    c, _ = h.cache(gpu)
    q = bf16(few, gpu)[torch.from_numpy(which).to(gpu)]
    out = torch.full(q.shape, float("nan"), device=gpu)
    wk.wushkv_cross_attention(c, q, f32(t, gpu), dev_i32(n_tok, gpu), dev_i32(np.where(source == 12, -1, source), gpu), out=out)
    live = np.arange(tok) < n_tok[:, None]
    if n * tok <= 20000:
        check(out.cpu().numpy(), np.where(live[..., None, None], want[source[:, None], which], 0.0),
              np.where(live[..., None], s[source[:, None], which], 0.0))
        return
    at = torch.from_numpy(np.where(live, source[:, None] * 7 + which, 12 * 7)).to(gpu)  # (the last is zeros)
    e = (out - torch.from_numpy(want.reshape(-1, hk * G, d)).to(gpu)[at]).norm(dim=-1)
    may = torch.from_numpy(3.0 * s.reshape(-1, hk * G)).to(gpu)[at]
    say("  rows' errors at most %.2f of what may be" % float((e[may > 0] / may[may > 0]).max()))
    assert bool((e <= may).all())
