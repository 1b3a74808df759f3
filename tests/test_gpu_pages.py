"""Boxes, selection, assignment and compaction of pages against their plain
forms (tests/pages_ref.py), value for value: every result is a whole number, a
moved byte or a value whose every step is one rounded operation."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
from gpu_harness import say
from pages_ref import Host
from workloads import synth

pytestmark = pytest.mark.gpu


def dev_i32(a, gpu):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(gpu)


def bf16(bits, gpu):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(gpu).view(torch.bfloat16)


def boxes_of(host):
    codes = np.zeros((host.n_pages, host.hk, 2, host.d), np.int8)
    scales = np.zeros((host.hk, host.n_pages), np.float32)
    return codes, scales


# ------------------------------------------------------------------ boxes


@pytest.mark.parametrize("d,bits,hk", [(64, 2, 1), (64, 4, 3), (128, 2, 5), (128, 4, 2), (128, 3, 1), (64, 3, 2)])
def test_boxes(gpu, d, bits, hk):
    say("boxes d %d, %d-bit, %d heads" % (d, bits, hk))
    rng = np.random.default_rng([d, bits, hk])
    # one token, none quantised, one page short of a token, one page, several
    h = Host(rng, [1, 36, 4 + 32 + 63, 4 + 32 + 64, 333, 500], hk, d, bits)
    since = np.array([0, 0, 0, 0, 4 + 64 + 5, 4 + 128], np.int32)
    # a page of zeros, one page with an infinite scale, one with a NaN zero
    par = h.pages.shape[2] - 512
    h.pages[h.table[4, 1], 0] = 0
    h.pages[h.table[4, 2], :, par + 8:par + 10] = np.array([0x00, 0x7C], np.uint8)
    h.pages[h.table[5, 3], :, par + 14:par + 16] = np.array([0x01, 0xFE], np.uint8)
    h.table[5, 5] = h.n_pages + 7  # outside the pool: skipped
    for use_since, most in ((False, None), (True, None), (True, 1), (False, 2)):
        c, _ = h.cache(gpu)
        b = wk.WushKVBounds(c)
        b.codes.fill_(77)
        b.scales.fill_(-3.0)
        codes, scales = boxes_of(h)
        codes[:], scales[:] = 77, -3.0
        for i in range(h.b):
            first = max(int(since[i]) - 4, 0) // 64 if use_since else 0
            for lp in range(first, min(h.complete(i), first + (h.max_pages if most is None else most))):
                p = h.table[i, lp]
                for k in range(hk):
                    if 0 <= p < h.n_pages:
                        codes[p, k], scales[k, p] = pages_ref.box(h.stored(p, k))
        wk.wushkv_page_bounds(c, b, since=dev_i32(since, gpu) if use_since else None, max_new=most)
        torch.cuda.synchronize()
        assert np.array_equal(b.scales.cpu().numpy(), scales)
        assert np.array_equal(b.codes.cpu().numpy(), codes)
        assert np.array_equal(c.pages.cpu().numpy(), h.pages.reshape(-1))


# ------------------------------------------------------------------ selection


def random_boxes(rng, host):
    codes, scales = boxes_of(host)
    codes[:, :, 0] = rng.integers(-100, 101, codes[:, :, 0].shape)
    codes[:, :, 1] = rng.integers(0, 27, codes[:, :, 1].shape)
    scales[:] = rng.uniform(0.01, 0.3, scales.shape)
    return codes, scales


def check_selection(gpu, host, codes, scales, q, t, top_k, **kw):
    c, _ = host.cache(gpu)
    b = wk.WushKVBounds(c)
    b.codes.copy_(torch.from_numpy(codes))
    b.scales.copy_(torch.from_numpy(scales))
    out = torch.full((host.b, host.hk, host.max_pages), 5.0, device=gpu)
    qd, td = bf16(q, gpu), torch.from_numpy(t).to(gpu)
    for s in (out, None):  # scores asked for and not
        sel, n = wk.wushkv_select_pages(c, b, qd, td, top_k, scores=s, **kw)
        torch.cuda.synchronize()
        ref = pages_ref.scores(host, codes, scales, q, t)
        rsel, rn = pages_ref.select(host, ref, top_k)
        assert np.array_equal(n.cpu().numpy(), rn)
        assert np.array_equal(sel.cpu().numpy(), rsel)
    # (entries behind the complete pages are left as they were)
    assert np.array_equal(out.cpu().numpy(), np.where(np.isnan(ref), np.float32(5.0), ref))


@pytest.mark.parametrize("d,G,hk,top_k", [(64, 1, 1, 0), (64, 2, 3, 1), (64, 8, 2, 3), (128, 1, 2, 4), (128, 4, 5, 2),
                                          (128, 8, 1, 7), (128, 2, 2, 40), (64, 4, 8, 5)])
def test_selection(gpu, d, G, hk, top_k):
    say("selection d %d, G %d, %d heads, top %d" % (d, G, hk, top_k))
    rng = np.random.default_rng([d, G, hk, top_k])
    h = Host(rng, [0, 1, 36, 99, 100, 333, 650], hk, d, 2)
    codes, scales = random_boxes(rng, h)
    q = synth.to_bf16_bits(rng.standard_normal((h.b, hk * G, d)))
    t = pages_ref.transform(rng, hk, d)
    check_selection(gpu, h, codes, scales, q, t, top_k)
    check_selection(gpu, h, codes, scales, q, t, top_k, max_seq_len=650)


def test_selection_takes_the_lowest_of_equals(gpu):
    rng = np.random.default_rng(31)
    h = Host(rng, [1500, 900], 2, 64, 2)
    codes, scales = random_boxes(rng, h)
    codes[:], scales[:] = codes[:1], scales[:, :1]  # every box the same
    q = synth.to_bf16_bits(rng.standard_normal((2, 4, 64)))
    t = pages_ref.transform(rng, 2, 64)
    for top_k in (1, 5, 12, 21, 22, 23):
        check_selection(gpu, h, codes, scales, q, t, top_k)
    # a few larger among them
    codes2 = codes.copy()
    codes2[h.table[0, [3, 17]], :, 1] += 3
    for top_k in (1, 2, 3, 9):
        check_selection(gpu, h, codes2, scales, q, t, top_k)


def test_selection_of_odd_values(gpu):
    rng = np.random.default_rng(32)
    h = Host(rng, [1000, 700, 640, 500], 2, 128, 4)
    codes, scales = random_boxes(rng, h)
    scales[:, h.table[0, 5]] = np.inf        # not finite: first
    codes[h.table[0, 5]] = 0
    scales[1, h.table[1, 2]] = 0.0           # a page of zeros
    codes[h.table[1, 2], 1] = 0
    h.table[2, 3] = -1                       # outside the pool: last
    h.table[2, 4] = h.n_pages
    codes[h.table[3], :, 1] = 0              # negative scores too
    q = rng.standard_normal((4, 4, 128)).astype(np.float32)
    q[0, 1] = 0.0                            # a query of zeros
    q[1, 2, 7] = np.nan
    q[1, 3, 9] = np.inf
    q[2] *= 1e30
    q[3] *= 1e-30
    t = pages_ref.transform(rng, 2, 128)
    for top_k in (1, 3, 8, 14):
        check_selection(gpu, h, codes, scales, synth.to_bf16_bits(q), t, top_k)


@pytest.mark.parametrize("pages,top_k", [(130, 17), (1000, 128), (2100, 64), (5000, 1000)])
def test_selection_of_many_pages(gpu, pages, top_k):
    say("selection of %d pages, top %d" % (pages, top_k))
    rng = np.random.default_rng(pages)
    lens = [4 + 32 + 64 * pages + 9, 64 * pages // 3 + 50]
    # the pages themselves are not read: all entries name a page of a small pool
    h = Host(rng, [200], 2, 64, 2, spare=60)
    h.b, h.seq_len = 2, np.asarray(lens, np.int32)
    h.quant_end = (4 + (h.seq_len - 36) // 8 * 8).astype(np.int32)
    h.max_pages = pages + 1
    h.table = rng.integers(0, h.n_pages, (2, h.max_pages)).astype(np.int32)
    h.held = np.full(2, h.max_pages, np.int32)
    h.win_k = np.repeat(h.win_k, 2, 0)
    h.win_v = np.repeat(h.win_v, 2, 0)
    codes, scales = random_boxes(rng, h)
    q = synth.to_bf16_bits(rng.standard_normal((2, 8, 64)))
    check_selection(gpu, h, codes, scales, q, pages_ref.transform(rng, 2, 64), top_k)


# ------------------------------------------------------------------ assignment


def same_state(c, pool, h):
    assert np.array_equal(c.page_table.cpu().numpy(), h.table)
    assert np.array_equal(pool.refs.cpu().numpy(), h.refs)
    assert np.array_equal(pool.held.cpu().numpy(), h.held)
    assert np.array_equal(c.seq_len.cpu().numpy(), h.seq_len)
    assert np.array_equal(c.quant_end.cpu().numpy(), h.quant_end)
    assert np.array_equal(c.win_k.view(torch.int16).cpu().numpy().view(np.uint16), h.win_k)
    assert np.array_equal(c.win_v.view(torch.int16).cpu().numpy().view(np.uint16), h.win_v)
    assert np.array_equal(c.pages.cpu().numpy(), h.pages.reshape(-1))
    low = int(pool.low.cpu()[0])
    assert (h.refs[:low] > 0).all()


@pytest.mark.parametrize("d,bits,hk", [(64, 2, 1), (128, 4, 3), (128, 3, 2)])
def test_assignment(gpu, d, bits, hk):
    say("assignment d %d, %d-bit, %d heads" % (d, bits, hk))
    rng = np.random.default_rng([d, bits, hk])
    h = Host(rng, [0, 20, 99, 100, 333, 421, 164, 650], hk, d, bits, spare=6, max_pages=12)
    c, pool = h.cache(gpu)
    steps = [
        (None, None),                                          # nothing
        (None, [0, 69, 5, 900, 333, 421, -7, 650]),            # pages for some
        ([0, 1, 2, 3, 4, 5, 6, 4], None),                      # one fork
        ([4, -1, 4, 3, 4, 3, 9, 3], [0, 300, 0, 0, 0, 0, 0, 0]),  # forks, a freed one that starts again, one refused
        ([0, -1, 1, 2, 4, 4, -2, 7], None),                    # sources that are not kept
        ([-1] * 8, None),                                      # everything freed
        (None, [800] * 8),                                     # more than there is
        ([7, 1, 1, 1, -1, -1, 0, 7], [0, 0, 900, 0, 100, 200, 700, 0]),
    ]
    for source, reach in steps:
        status = wk.wushkv_assign_pages(c, pool, source=None if source is None else dev_i32(source, gpu),
                                        reach=None if reach is None else dev_i32(reach, gpu))
        torch.cuda.synchronize()
        want = pages_ref.assign(h, source, reach)
        assert np.array_equal(status.cpu().numpy(), want), (source, reach)
        same_state(c, pool, h)


@pytest.mark.parametrize("seed", range(6))
def test_assignment_over_many_steps(gpu, seed):
    """Random calls on a tight pool, and now and then a compaction, in place
    or not."""
    rng = np.random.default_rng([seed, 77])
    B = int(rng.integers(2, 40))
    h = Host(rng, rng.integers(0, 700, B), int(rng.integers(1, 3)), 64, 2, spare=int(rng.integers(0, 20)), max_pages=11)
    c, pool = h.cache(gpu)
    bounds = wk.WushKVBounds(c)
    codes, scales = random_boxes(rng, h)
    bounds.codes.copy_(torch.from_numpy(codes))
    bounds.scales.copy_(torch.from_numpy(scales))
    for step in range(12):
        if rng.random() < 0.3:
            if rng.random() < 0.5:
                t, r, n = wk.wushkv_compact_pages(c, pool, bounds=bounds)
            else:
                old = c.page_table.clone(), pool.refs.clone()
                t, r, n = wk.wushkv_compact_pages(c, pool, bounds=bounds, table_out=torch.empty_like(c.page_table),
                                                  refs_out=torch.empty_like(pool.refs))
                torch.cuda.synchronize()
                assert torch.equal(c.page_table, old[0]) and torch.equal(pool.refs, old[1])
                c.page_table.copy_(t)
                pool.refs.copy_(r)
            assert int(n.cpu()[0]) == pages_ref.compact(h, codes, scales)
            # (a page that moved is left where it was, as its own old copy)
        else:
            source = np.where(rng.random(B) < 0.6, np.arange(B), rng.integers(-2, B + 1, B))
            reach = rng.integers(0, 900, B) * (rng.random(B) < 0.4)
            status = wk.wushkv_assign_pages(c, pool, source=dev_i32(source, gpu), reach=dev_i32(reach, gpu))
            want = pages_ref.assign(h, source, reach)
            assert np.array_equal(status.cpu().numpy(), want), step
        torch.cuda.synchronize()
        same_state(c, pool, h)
        assert np.array_equal(bounds.codes.cpu().numpy(), codes) and np.array_equal(bounds.scales.cpu().numpy(), scales)


def test_large_batches_and_pools(gpu):
    """More sequences than a workgroup has threads, and more pages than one of
    its rounds or a block of references covers."""
    B, n = 1500, 20011
    c = wk.WushKVCache(B, 1, 64, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=4 + 64 * 20, win_slots=64, page_order="none",
                       n_pages=n, device=gpu)
    pool = wk.WushKVPool(c)
    rng = np.random.default_rng(8)
    taken = rng.random(n) < 0.3
    pool.refs.copy_(torch.from_numpy(taken.astype(np.int32)))
    want = rng.integers(0, 14, B)
    status = wk.wushkv_assign_pages(c, pool, reach=dev_i32(np.where(want > 0, 4 + 64 * want, 0), gpu)).cpu().numpy()
    free = np.flatnonzero(~taken)
    start = np.cumsum(want) - want
    got = np.clip(len(free) - start, 0, want)
    assert np.array_equal(status, want - got) and np.array_equal(pool.held.cpu().numpy(), got)
    table = c.page_table.cpu().numpy()
    for b in range(B):
        assert np.array_equal(table[b, :got[b]], free[start[b]:start[b] + got[b]])
        assert (table[b, got[b]:] == -1).all()
    # every other sequence ends; the rest moves to the front
    source = np.where(np.arange(B) % 2 == 0, np.arange(B), -1)
    wk.wushkv_assign_pages(c, pool, source=dev_i32(source, gpu))
    c.pages.view(n, -1)[:, :4].copy_(torch.arange(n, device=gpu, dtype=torch.int32).view(n, 1).view(torch.uint8))
    before = c.page_table.clone()
    live = int((pool.refs > 0).sum())
    _, _, count = wk.wushkv_compact_pages(c, pool)
    assert int(count[0]) == live and bool((pool.refs[:live] > 0).all()) and not bool(pool.refs[live:].any())
    after, names = c.page_table, c.pages.view(n, -1)[:, :4].contiguous().view(torch.int32)[:, 0]
    there = before >= 0
    assert torch.equal(after >= 0, there) and int(after.max()) < live
    assert torch.equal(names[after[there].long()], before[there])


def test_pages_beyond_four_gigabytes(gpu):
    """Physical pages whose bytes lie past 2^32."""
    say("pages beyond 4 GiB")
    rng = np.random.default_rng(12)
    h = Host(rng, [300], 8, 128, 4)
    n = (1 << 32) // (8 * h.pages.shape[2]) + 40
    c = wk.WushKVCache(1, 8, 128, 4, 4, 32, 8, 0.96, 0.92, max_seq_len=4 + 64 * h.max_pages, win_slots=64,
                       page_order="none", n_pages=n, device=gpu)
    k = len(h.used)
    far = torch.from_numpy(np.arange(n - k, n)).to(gpu)
    place = {int(p): n - k + i for i, p in enumerate(h.used)}
    c.pages.view(n, 8, -1)[far] = torch.from_numpy(h.pages[h.used]).to(gpu)
    c.page_table.copy_(torch.from_numpy(np.vectorize(lambda p: place.get(int(p), -1))(h.table).astype(np.int32)))
    c.seq_len.copy_(torch.from_numpy(h.seq_len))
    c.quant_end.copy_(torch.from_numpy(h.quant_end))
    pool, b = wk.WushKVPool(c), wk.WushKVBounds(c)
    wk.wushkv_page_bounds(c, b)
    codes, scales = b.codes[far].cpu().numpy(), b.scales[:, far].cpu().numpy()
    for lp in range(h.complete(0)):
        i = place[int(h.table[0, lp])] - (n - k)
        for head in range(8):
            want = pages_ref.box(h.stored(h.table[0, lp], head))
            assert np.array_equal(codes[i, head], want[0]) and scales[head, i] == want[1]
    wk.wushkv_compact_pages(c, pool, bounds=b)
    assert torch.equal(c.pages.view(n, 8, -1)[:k].cpu(), torch.from_numpy(h.pages[h.used]))
    assert np.array_equal(b.codes[:k].cpu().numpy(), codes) and np.array_equal(b.scales[:, :k].cpu().numpy(), scales)


def test_forks_and_compactions_replayed(gpu):
    """Frees, forks, extensions and a compaction captured once and replayed with
    other source maps, against the plain forms, value for value."""
    rng = np.random.default_rng(51)
    h = Host(rng, rng.integers(0, 600, 12), 2, 64, 2, spare=25, max_pages=10)
    c, pool = h.cache(gpu)
    source, reach = torch.zeros(12, dtype=torch.int32, device=gpu), torch.zeros(12, dtype=torch.int32, device=gpu)
    bounds = wk.WushKVBounds(c)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        status = wk.wushkv_assign_pages(c, pool, source=source, reach=reach)
        wk.wushkv_page_bounds(c, bounds)
        _, _, live = wk.wushkv_compact_pages(c, pool, bounds=bounds)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(6):
        src = np.where(rng.random(12) < 0.5, np.arange(12), rng.integers(-1, 12, 12))
        want = rng.integers(0, 640, 12) * (rng.random(12) < 0.3)
        source.copy_(dev_i32(src, gpu))
        reach.copy_(dev_i32(want, gpu))
        if i % 2:
            torch.cuda.synchronize()
        graph.replay()
        expect = pages_ref.assign(h, src, want)
        n = pages_ref.compact(h)
        torch.cuda.synchronize()
        assert np.array_equal(status.cpu().numpy(), expect) and int(live[0]) == n
        same_state(c, pool, h)
        for b in range(h.b):
            for lp in range(min(h.complete(b), int(h.held[b]))):
                p = h.table[b, lp]
                codes, scale = pages_ref.box(h.stored(p, 1))
                assert np.array_equal(bounds.codes[p, 1].cpu().numpy(), codes) and float(bounds.scales[1, p]) == scale
