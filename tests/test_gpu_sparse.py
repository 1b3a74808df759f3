"""Attention over listed pages against a plain 64-bit evaluation, within the
bound that pages_ref.attention derives, and against the dense decode; then
the page operators and the attention together, as a serving loop runs them."""
import numpy as np
import pytest
import torch

import oracle
import pages_ref
import paper_2609_38121_amd as wk
from gpu_harness import Pair, TOL, rel_err, say, to_dev_bf16
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from workloads import synth

pytestmark = pytest.mark.gpu


def run(gpu, host, q, t, sel, n_sel, cache=None):
    c = cache or host.cache(gpu)[0]
    out = torch.full((host.b, q.shape[1], host.d), float("nan"), device=gpu)
    wk.wushkv_sparse_attention(c, bf16(q, gpu), torch.from_numpy(t).to(gpu), dev_i32(sel, gpu), dev_i32(n_sel, gpu), out=out)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def check(gpu, host, q, t, sel, n_sel):
    got = run(gpu, host, q, t, sel, n_sel)
    want, tol = pages_ref.attention(host, q, t, sel, n_sel, 1.0 / np.sqrt(host.d))
    off = np.abs(got - want).max(-1)
    say("  largest error %.2e, of its bound %.2f" % (off.max(), (off / np.maximum(tol, 1e-30)).max()))
    assert (off <= tol).all()
    return got


def lists(rng, host, width):
    """Random pages in random order, some with the one being filled."""
    sel = np.full((host.b, host.hk, width), -1, np.int32)
    n = np.zeros((host.b, host.hk), np.int32)
    for b in range(host.b):
        for h in range(host.hk):
            k = int(rng.integers(0, min(width, host.every(b)) + 1))
            sel[b, h, :k] = rng.permutation(host.every(b))[:k]
            n[b, h] = k
    return sel, n


@pytest.mark.parametrize("d,bits,G,hk", [(64, 2, 1, 2), (64, 4, 4, 1), (64, 2, 8, 1), (64, 3, 2, 3), (128, 2, 4, 2),
                                         (128, 4, 8, 1), (128, 4, 1, 5), (128, 2, 8, 2), (128, 3, 2, 1), (64, 4, 8, 2),
                                         (128, 2, 1, 1), (128, 4, 4, 2)])
def test_listed_pages(gpu, d, bits, G, hk):
    say("sparse d %d, %d-bit, G %d, %d heads" % (d, bits, G, hk))
    rng = np.random.default_rng([d, bits, G, hk])
    # nothing, one token, the sink alone, windows alone, a part of a page, several pages
    h = Host(rng, [0, 1, 4, 36, 45, 100, 333, 700], hk, d, bits)
    # dead slots and the rows of the page being filled hold NaN patterns
    for b in range(h.b):
        S, end = int(h.seq_len[b]), h.end(b)
        live = [p if p < 4 else 4 + (p - 4) % 60 for p in range(S) if p < 4 or p >= end]
        dead = np.setdiff1d(np.arange(64), live)
        h.win_k[b][:, dead] = 0x7FC1
        h.win_v[b][:, :, dead] = 0xFFFF
        if h.every(b) > h.complete(b):
            first = end - 4 - 64 * h.complete(b)
            par = h.pages.shape[2] - 512
            page = h.pages[h.table[b, h.complete(b)]]
            page[:, par + 4 * first:par + 256] = 0xFF
            page[:, par + 256 + 4 * first:] = 0xFF
    q = synth.to_bf16_bits(rng.standard_normal((h.b, hk * G, d)))
    t = pages_ref.transform(rng, hk, d)
    for width in (1, 4, 11):
        sel, n = lists(rng, h, width)
        check(gpu, h, q, t, sel, n)
    # every page: what the dense decode attends to
    every = max(h.every(b) for b in range(h.b))
    sel = np.broadcast_to(np.arange(every, dtype=np.int32), (h.b, hk, every)).copy()
    n = np.repeat(np.array([h.every(b) for b in range(h.b)], np.int32)[:, None], hk, 1)
    got = check(gpu, h, q, t, sel, n)
    assert (got[0] == 0).all()
    c, _ = h.cache(gpu)
    dense = wk.wushkv_decode_attention(c, bf16(q, gpu), torch.from_numpy(t).to(gpu)).cpu().numpy()
    # (the dense decode takes q~ to two bf16 parts over the windows)
    assert rel_err(got, dense) <= 1e-3


def test_odd_lists(gpu):
    rng = np.random.default_rng(21)
    h = Host(rng, [600, 350, 90], 2, 128, 2)
    q = synth.to_bf16_bits(rng.standard_normal((3, 4, 128)))
    t = pages_ref.transform(rng, 2, 128)
    none = np.zeros((3, 2), np.int32)
    # an empty list, of width 0 and 3
    check(gpu, h, q, t, np.zeros((3, 2, 0), np.int32), none)
    check(gpu, h, q, t, np.full((3, 2, 3), 1, np.int32), none)
    # entries outside the table, pages behind the end, counts outside [0, width]
    sel = np.array([[[2, -5, 1 << 30, 0], [5, 5, 1, -1]], [[4, 3, 0, 9999], [1, 2, 3, 0]], [[0, 1, 2, 3], [-1, -1, -1, -1]]],
                   np.int32)
    check(gpu, h, q, t, sel, np.array([[4, 3], [4, 900], [4, -3]], np.int32))
    # a page outside the pool
    h.table[0, 2] = h.n_pages
    h.table[1, 3] = -9
    check(gpu, h, q, t, sel, np.full((3, 2), 4, np.int32))


@pytest.mark.parametrize("batch,hk,G,bits,width", [(70, 8, 4, 2, 6), (40, 8, 8, 4, 5), (3, 2, 4, 2, 200)])
def test_grids_of_rounds_and_long_lists(gpu, batch, hk, G, bits, width):
    """More workgroups than the device keeps at once, and lists over several
    runs: pages of a small pool, many rows naming the same."""
    say("sparse batch %d, %d heads, G %d, %d-bit, %d pages" % (batch, hk, G, bits, width))
    rng = np.random.default_rng(batch)
    h = Host(rng, [1200], hk, 128, bits, s_keep=100, win_slots=192)
    first = h.table[0, :h.complete(0)].copy()
    h.b, h.max_pages = batch, width + 1
    h.seq_len = rng.integers(64 * width // 2 + 200, 64 * width + 200, batch).astype(np.int32)
    h.quant_end = (4 + (h.seq_len - 104) // 8 * 8).astype(np.int32)
    h.table = rng.choice(first, (batch, h.max_pages)).astype(np.int32)
    h.held = np.full(batch, h.max_pages, np.int32)
    h.win_k = rng.permuted(np.repeat(h.win_k, batch, 0), axis=2)
    h.win_v = np.repeat(h.win_v, batch, 0)
    q = synth.to_bf16_bits(rng.standard_normal((batch, hk * G, 128)))
    t = pages_ref.transform(rng, hk, 128)
    sel, n = lists(rng, h, width)
    if batch == 3:  # the plain evaluation of long lists for a few rows
        check(gpu, h, q, t, sel, n)
        return
    got = run(gpu, h, q, t, sel, n)
    pick = rng.choice(batch, 4, replace=False)
    want, tol = pages_ref.attention(some(h, pick), q[pick], t, sel[pick], n[pick], 1.0 / np.sqrt(128))
    assert (np.abs(got[pick] - want).max(-1) <= tol).all()
    # the same call again: the same bits
    assert np.array_equal(run(gpu, h, q, t, sel, n), got)


def some(host, pick):
    """The state of some of a host's sequences."""
    part = object.__new__(Host)
    part.__dict__.update(host.__dict__)
    part.b = len(pick)
    for name in ("seq_len", "quant_end", "table", "win_k", "win_v"):
        setattr(part, name, getattr(host, name)[pick])
    return part


@pytest.mark.parametrize("d,bits,G,slots", [(128, 2, 1, 64), (128, 4, 2, 64), (128, 2, 8, 128), (128, 4, 8, 64), (64, 2, 8, 64),
                                            (64, 4, 2, 192), (128, 3, 4, 64)])
def test_a_row_for_every_compute_unit(gpu, d, bits, G, slots):
    """Batches whose rows are one workgroup's each, lists of no page to more
    than there are."""
    say("sparse, whole rows: d %d, %d-bit, G %d, %d slots" % (d, bits, G, slots))
    rng = np.random.default_rng([d, bits, G, slots])
    lens = rng.integers(0, 330, 150)
    lens[:8] = [0, 1, 4, 5, 36, 45, 100, 329]
    h = Host(rng, lens, 2, d, bits, win_slots=slots)
    q = synth.to_bf16_bits(rng.standard_normal((h.b, 2 * G, d)))
    t = pages_ref.transform(rng, 2, d)
    pick = np.concatenate([np.arange(8), rng.choice(np.arange(8, 150), 5, replace=False)])
    for width in (0, 3, 70):
        sel, n = lists(rng, h, width) if width < 70 else (rng.integers(-1, 5, (h.b, 2, 70)).astype(np.int32),
                                                          rng.integers(0, 80, (h.b, 2)).astype(np.int32))
        got = run(gpu, h, q, t, sel, n)
        want, tol = pages_ref.attention(some(h, pick), q[pick], t, sel[pick], n[pick], 1.0 / np.sqrt(d))
        off = np.abs(got[pick] - want).max(-1)
        say("  width %d: of its bound %.2f" % (width, (off / np.maximum(tol, 1e-30)).max()))
        assert (off <= tol).all() and np.isfinite(got).all()


@pytest.mark.parametrize("batch,d,bits", [(2, 128, 4), (2, 64, 2), (140, 128, 2)])
def test_large_value_scales(gpu, batch, d, bits):
    """Values far larger in some pages than in others: weights times scales
    beyond fp16 if they were lifted everywhere."""
    rng = np.random.default_rng([batch, d, bits])
    h = Host(rng, [700] * 2 + [50] * (batch - 2), 2, d, bits)
    par = h.pages.shape[2] - 256
    for lp, scale in ((1, 150.0), (4, 30000.0), (7, 127.0), (9, 60000.0)):
        for b in range(2):
            view = h.pages[h.table[b, lp], :, par:].view(np.float16).reshape(2, 64, 2)
            view[:, :, 0] = scale
            h.pages[h.table[b, lp], :, par:] = view.reshape(2, 128).view(np.uint8)
    q = synth.to_bf16_bits(rng.standard_normal((h.b, 4, d)))
    t = pages_ref.transform(rng, 2, d)
    for _ in range(3):
        sel, n = lists(rng, h, 10)
        got = run(gpu, h, q, t, sel, n)
        pick = np.arange(min(batch, 4))
        want, tol = pages_ref.attention(some(h, pick), q[pick], t, sel[pick], n[pick], 1.0 / np.sqrt(d))
        assert (np.abs(got[pick] - want).max(-1) <= tol).all()


@pytest.mark.parametrize("s_sink,win_slots,s_keep,s_flush", [(0, 64, 32, 8), (70, 128, 32, 5), (9, 256, 180, 16), (0, 64, 0, 1)])
@pytest.mark.parametrize("batch", [5, 140])
def test_other_windows(gpu, s_sink, win_slots, s_keep, s_flush, batch):
    """Boxes, selection, attention and forks with no sink, one that spans tiles,
    and long rings."""
    rng = np.random.default_rng([s_sink, win_slots, batch])
    lens = np.concatenate([[0, 1, s_sink, s_sink + s_keep + 1, 400], rng.integers(0, 60, batch - 5)])
    h = Host(rng, lens, 2, 128, 2, s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, win_slots=win_slots, spare=12, max_pages=8)
    q = synth.to_bf16_bits(rng.standard_normal((batch, 4, 128)))
    t = pages_ref.transform(rng, 2, 128)
    c, pool = h.cache(gpu)
    bounds = wk.WushKVBounds(c)
    codes, scales = np.zeros((h.n_pages, 2, 2, 128), np.int8), np.zeros((2, h.n_pages), np.float32)
    for b in range(5):
        for lp in range(h.complete(b)):
            for k in range(2):
                codes[h.table[b, lp], k], scales[k, h.table[b, lp]] = pages_ref.box(h.stored(h.table[b, lp], k))
    pick = np.arange(5)
    for _ in range(2):  # as it is, and with the long sequence forked into two others
        wk.wushkv_page_bounds(c, bounds)
        sel, n = wk.wushkv_select_pages(c, bounds, bf16(q, gpu), torch.from_numpy(t).to(gpu), 3)
        few = some(h, pick)
        rsel, rn = pages_ref.select(few, pages_ref.scores(few, codes, scales, q[pick], t), 3)
        sel, n = sel.cpu().numpy(), n.cpu().numpy()
        assert np.array_equal(sel[pick], rsel) and np.array_equal(n[pick], rn)
        got = run(gpu, h, q, t, sel, n, cache=c)
        want, tol = pages_ref.attention(few, q[pick], t, sel[pick], n[pick], 1.0 / np.sqrt(128))
        assert (np.abs(got[pick] - want).max(-1) <= tol).all()
        source = np.arange(batch)
        source[[0, 2]] = 4
        status = wk.wushkv_assign_pages(c, pool, source=dev_i32(source, gpu))
        assert np.array_equal(status.cpu().numpy(), pages_ref.assign(h, source))


# ------------------------------------------------------------------ together


def kv(rng, B, n, H, d):
    k = rng.standard_normal((B, n, H, d)).astype(np.float32)
    k[..., [5, 40]] *= 8.0
    return oracle.f32_to_bf16(k), oracle.f32_to_bf16(rng.standard_normal((B, n, H, d)).astype(np.float32))


@pytest.mark.parametrize("d,bits,G,codec", [(64, 2, 4, "pclip"), (128, 4, 2, "quest")])
def test_a_serving_loop(gpu, d, bits, G, codec):
    """Prompts into pages that the pool hands out, decode steps with growing
    boxes and selected pages, forks that then go their own ways, frees and a
    compaction.  Selecting every page gives the dense decode; a fork's rows are
    those of a sequence that was never forked; a compaction changes nothing."""
    say("serving loop d %d, %d-bit, %s" % (d, bits, codec))
    rng = np.random.default_rng([d, bits])
    B, H, cap = 5, 2, 900
    p = Pair(gpu, B, H, G, d, bits, 4, 64, 8, 0.96, 0.92, cap=cap, oracle_ref=False, codec=codec)
    c = wk.WushKVCache(B, H, d, bits, 4, 64, 8, 0.96, 0.92, max_seq_len=cap, device=gpu, codec=codec,
                       quest_alpha=p.gpu.quest_alpha if codec == "quest" else None, page_order="none", n_pages=40)
    plain, p.gpu = p.gpu, c  # the oracle's cache follows this one; `plain` never shares a page
    pool, bounds = wk.WushKVPool(c), wk.WushKVBounds(c)
    lens = np.array([700, 333, 0, 520, 0], np.int32)
    assert not wk.wushkv_assign_pages(c, pool, reach=dev_i32(lens, gpu)).any()
    k, v = kv(rng, B, 700, H, d)
    p.append(k, v, lens)
    args = to_dev_bf16(k, gpu), to_dev_bf16(v, gpu), dev_i32(lens, gpu), p.tk_dev
    wk.wushkv_append(plain, *args)
    wk.wushkv_page_bounds(c, bounds)

    def attend(top_k, tol):
        q = oracle.f32_to_bf16(rng.standard_normal((B, H * G, d)).astype(np.float32))
        sel, n = wk.wushkv_select_pages(c, bounds, to_dev_bf16(q, gpu), p.tinv_dev, top_k)
        out = wk.wushkv_sparse_attention(c, to_dev_bf16(q, gpu), p.tinv_dev, sel, n).cpu().numpy()
        dense = wk.wushkv_decode_attention(c, to_dev_bf16(q, gpu), p.tinv_dev)
        other = wk.wushkv_decode_attention(plain, to_dev_bf16(q, gpu), p.tinv_dev)
        assert torch.equal(dense, other)
        assert rel_err(out, dense.cpu().numpy()) <= tol
        return out

    attend(cap // 64, 1e-3)
    attend(2, np.inf)

    def steps(count):
        since = c.quant_end.clone()
        assert not wk.wushkv_assign_pages(c, pool, reach=c.seq_len + count * (c.seq_len > 0).int()).any()
        for _ in range(count):
            k1, v1 = kv(rng, B, 1, H, d)
            n1 = (c.seq_len > 0).int()
            for cache in (c, plain):
                wk.wushkv_append(cache, to_dev_bf16(k1, gpu), to_dev_bf16(v1, gpu), n1, p.tk_dev)
        wk.wushkv_page_bounds(c, bounds, since=since)
        rebuilt = wk.WushKVBounds(c)
        wk.wushkv_page_bounds(c, rebuilt)
        live = [c.page_table[b, lp] for b in range(B) for lp in range(max(int(c.quant_end[b]) - 4, 0) // 64)]
        at = torch.stack(live).long()
        assert torch.equal(rebuilt.codes[at], bounds.codes[at]) and torch.equal(rebuilt.scales[:, at], bounds.scales[:, at])

    def copy(src, dst):  # on the cache that never shares
        pages = plain.pages.view(plain.n_pages, -1)
        pages[plain.page_table[dst].long()] = pages[plain.page_table[src].long()]
        for t in (plain.win_k, plain.win_v, plain.seq_len, plain.quant_end):
            t[dst] = t[src]

    steps(70)
    attend(cap // 64, 1e-3)
    # 2 and 4 become copies of 0 and 3
    assert not wk.wushkv_assign_pages(c, pool, source=dev_i32([0, 1, 0, 3, 3], gpu)).any()
    copy(0, 2)
    copy(3, 4)
    full = (int(c.quant_end[0]) - 4) // 64
    assert torch.equal(c.page_table[0, :full], c.page_table[2, :full])
    assert bool((pool.refs[c.page_table[0, :full].long()] == 2).all())
    attend(cap // 64, 1e-3)
    steps(21)
    attend(cap // 64, 1e-3)
    # 0 ends; its pages stay with 2
    assert not wk.wushkv_assign_pages(c, pool, source=dev_i32([-1, 1, 2, 3, 4], gpu)).any()
    plain.seq_len[0] = plain.quant_end[0] = 0
    attend(cap // 64, 1e-3)
    before = attend(3, np.inf).shape
    _, refs, live = wk.wushkv_compact_pages(c, pool, bounds=bounds)
    assert int(live[0]) == int((refs > 0).sum()) and int(c.page_table.max()) < int(live[0])
    attend(cap // 64, 1e-3)
    steps(9)
    assert attend(cap // 64, 1e-3).shape == before


def test_replayed_graphs_and_streams(gpu):
    """A whole step (pages, boxes, selection, attention) captured once and
    replayed over changing inputs, on a stream of its own, against eager calls
    on another cache; the program's own work between the replays."""
    rng = np.random.default_rng(41)
    B, H, G, d = 3, 2, 4, 128
    h = Host(rng, [900, 400, 120], H, d, 2, spare=30, max_pages=20)
    t = torch.from_numpy(pages_ref.transform(rng, H, d)).to(gpu)
    tk = torch.eye(d, dtype=torch.bfloat16, device=gpu).expand(H, d, d).contiguous()

    class Loop:
        def __init__(self):
            self.c, self.pool = h.cache(gpu)
            self.bounds = wk.WushKVBounds(self.c)
            wk.wushkv_page_bounds(self.c, self.bounds)
            self.k = torch.zeros(B, 9, H, d, dtype=torch.bfloat16, device=gpu)
            self.v, self.q = torch.zeros_like(self.k), torch.zeros(B, H * G, d, dtype=torch.bfloat16, device=gpu)
            self.n = torch.full((B,), 9, dtype=torch.int32, device=gpu)

        def step(self):
            since = self.c.quant_end.clone()
            self.status = wk.wushkv_assign_pages(self.c, self.pool, reach=self.c.seq_len + 9)
            wk.wushkv_append(self.c, self.k, self.v, self.n, tk)
            wk.wushkv_page_bounds(self.c, self.bounds, since=since, max_new=1)
            self.sel, self.count = wk.wushkv_select_pages(self.c, self.bounds, self.q, t, 3)
            self.out = wk.wushkv_sparse_attention(self.c, self.q, t, self.sel, self.count)

    eager, other = Loop(), Loop()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        other.step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(6):
        say("replay %d" % i)
        for name in ("k", "v", "q"):
            x = torch.from_numpy(rng.standard_normal(tuple(getattr(eager, name).shape)).astype(np.float32)).to(gpu)
            getattr(eager, name).copy_(x)
            getattr(other, name).copy_(x)
        eager.step()
        if i % 2:
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("status", "sel", "count", "out"):
            assert torch.equal(getattr(eager, name), getattr(other, name)), (i, name)
        assert torch.equal(eager.c.page_table, other.c.page_table)
        assert torch.equal(eager.bounds.codes, other.bounds.codes)
    # the same calls on a stream given by hand, buffers made inside
    sel0, n0 = wk.wushkv_select_pages(eager.c, eager.bounds, eager.q, t, 3)
    side.wait_stream(torch.cuda.current_stream())
    sel1, n1 = wk.wushkv_select_pages(eager.c, eager.bounds, eager.q, t, 3, stream=side)
    out1 = wk.wushkv_sparse_attention(eager.c, eager.q, t, sel1, n1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(sel0, sel1) and torch.equal(out1, wk.wushkv_sparse_attention(eager.c, eager.q, t, sel0, n0))


@pytest.mark.parametrize("d,bits,G", [(64, 2, 4), (128, 4, 2), (128, 2, 8), (64, 3, 8)])
def test_pages_that_held_something_else(gpu, d, bits, G):
    """Pages full of NaN patterns taken for new sequences: the same bits as
    from zeroed ones, from every attention that reads them."""
    rng = np.random.default_rng([d, bits, G, 5])
    lens = [301, 90, 64 + 4 + 40 + 3]
    H, B = 2, len(lens)
    p = Pair(gpu, B, H, G, d, bits, 4, 40, 8, 0.96, 0.92, cap=400, oracle_ref=False)
    other = p.gpu.clone()
    other.pages.fill_(255)
    k, v = kv(rng, B, max(lens), H, d)
    n = dev_i32(lens, gpu)
    q = to_dev_bf16(oracle.f32_to_bf16(rng.standard_normal((B, 17, H * G, d)).astype(np.float32)), gpu)
    k1, v1 = (to_dev_bf16(x[:, 0], gpu) for x in kv(rng, B, 1, H, d))
    got = []
    for c in (p.gpu, other):
        wk.wushkv_append(c, to_dev_bf16(k, gpu), to_dev_bf16(v, gpu), n, p.tk_dev)
        first = q[:, 0].contiguous()
        sel = torch.arange(5, device=gpu, dtype=torch.int32).expand(B, H, 5).contiguous()
        got.append([
            wk.wushkv_decode_attention(c, first, p.tinv_dev),
            wk.wushkv_chunk_attention(c, q, p.tinv_dev),
            wk.wushkv_sparse_attention(c, first, p.tinv_dev, sel, torch.full((B, H), 5, device=gpu, dtype=torch.int32)),
            wk.wushkv_decode_step(c, k1, v1, torch.ones_like(n), p.tk_dev, first, p.tinv_dev),
        ])
    for a, b in zip(*got):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
