"""Prefix, cross and weighted attention as they are used: on other streams, captured
and replayed, with workspaces that hold something else or are shared, over pools
of more than 4 GiB, in states that strain the arithmetic, and together with the
forks, the eviction, the page lists and the compaction of a serving loop."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
import rows_exact
import sparse_exact
from gpu_harness import say
from pages_ref import Host
from sparse_exact import params, put
from test_gpu_pages import bf16, dev_i32, same_state
from test_gpu_rows import f32, fork, queries, run_cross, run_prefix, run_weighted

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ states


@pytest.mark.parametrize("name", sorted(sparse_exact.STATES))
@pytest.mark.parametrize("d,bits,G,hk", [(128, 2, 4, 1), (64, 4, 8, 2), (128, 4, 1, 1), (64, 2, 2, 1)])
def test_states(gpu, name, d, bits, G, hk):
    say("%s, d %d, %d-bit, G %d" % (name, d, bits, G))
    h, q, t, sel, n = sparse_exact.state(name, d, bits, G, hk, 6, win_slots=128)
    rng = np.random.default_rng([d, bits, len(name)])
    run_weighted(gpu, h, q, t, rng.exponential(1.0, (6, hk, h.max_pages)))
    run_weighted(gpu, h, q, t, np.zeros((6, hk, h.max_pages)), sel, n)
    run_cross(gpu, h, np.stack([q, q[::-1], q], 1), t, None, np.array([2, 1, 0, 0, 5, 1]))
    if name != "windows":
        fork(h, 2, 0, 3)
        fork(h, 1, 0, 2)
    run_prefix(gpu, h, q, t, np.array([0, 0, 0, 3, 4, 5]), np.array([0, 2, 3, 0, 0, 0]))


@pytest.mark.parametrize("d,bits", [(128, 2), (64, 4)])
@pytest.mark.parametrize("name", ["zero", "tiny", "large", "rising", "falling", "windows"])
def test_values_of_any_size(gpu, name, d, bits):
    """Value scales of zero, subnormal, near the largest, and that change by powers of
    two from page to page; windows near the largest bf16 number."""
    say("%s, d %d, %d-bit" % (name, d, bits))
    rng = np.random.default_rng([d, bits, len(name)])
    h = Host(rng, [800, 333, 500], 2, d, bits)
    for b in range(3):
        for i in range(h.every(b)):
            x = params(h, h.table[b, i], True).copy()
            if name == "zero":          # every other page is all zeros' worth
                x[:, :, 0] *= i % 2
            if name == "tiny":          # 2^-24 .. 2^-20: subnormal
                x[:, :, 0] = rng.integers(1, 16, (2, 64)) * 2.0 ** -24
                x[:, :, 1] = 0.0
            if name == "large":
                x[:, :, 0], x[:, :, 1] = rng.uniform(3e4, 65504.0, (2, 64)), 0.0
            if name == "rising":
                x[:, :, 0] *= 2.0 ** (i - 8)
            if name == "falling":
                x[:, :, 0] *= 2.0 ** (5 - i)
            put(h, h.table[b, i], True, x)
    if name == "windows":
        h.win_v = pages_ref.synth.to_bf16_bits(rng.uniform(-3.3e38, 3.3e38, h.win_v.shape))
    q, t = queries(rng, 3, 8, d), pages_ref.transform(rng, 2, d)
    run_weighted(gpu, h, q, t, np.zeros((3, 2, h.max_pages)))
    run_cross(gpu, h, np.stack([q, q[::-1]], 1), t)
    fork(h, 1, 0, 4)
    run_prefix(gpu, h, q, t, np.array([0, 0, 2]), np.array([0, 4, 0]))


def test_rows_are_apart(gpu):
    """Queries that are not numbers spoil no other row of their tile."""
    rng = np.random.default_rng(11)
    h = Host(rng, [700, 650, 600, 500], 2, 128, 2)
    for b in (1, 2, 3):
        fork(h, b, 0, 6)
    q, t = queries(rng, 4, 8, 128), pages_ref.transform(rng, 2, 128)
    leader, shared = np.zeros(4, int), np.array([0, 6, 6, 6])
    want, s, w = rows_exact.prefix(h, q, t, leader, shared)
    bad = q.copy()
    bad[1, 2, :5] = [0x7FC0, 0x7F80, 0xFF80, 0x7FFF, 0x7F7F]
    c, _ = h.cache(gpu)
    got = wk.wushkv_prefix_attention(c, bf16(bad, gpu), f32(t, gpu), dev_i32(leader, gpu), dev_i32(shared, gpu)).cpu().numpy()
    keep = np.ones((4, 8), bool)
    keep[1, 2] = False
    assert rows_exact.off(got[keep], want[keep], s[keep], w[keep]) <= 1.0


# ------------------------------------------------------------------ streams, workspaces, graphs


class Calls:
    """The three attentions on one cache, with buffers of their own."""

    def __init__(self, gpu, seed, space=None):
        rng = np.random.default_rng(seed)
        self.h = h = Host(rng, [700, 333, 650, 0, 500, 1], 2, 128, 2, max_pages=12)
        for b, n in ((2, 7), (4, 3)):
            fork(h, b, 0, n)
        self.c, self.pool = h.cache(gpu)
        self.q, self.x = bf16(queries(rng, 6, 8, 128), gpu), bf16(queries(rng, 5, 3, 8, 128), gpu)
        self.t = f32(pages_ref.transform(rng, 2, 128), gpu)
        self.n_tok, self.source = dev_i32([3, 1, 2, 0, 3], gpu), dev_i32([0, 2, 4, 1, 0], gpu)
        self.weights = torch.zeros(6, 2, 12, device=gpu)
        need = max(wk.wushkv_prefix_workspace_bytes(self.c, 8), wk.wushkv_cross_workspace_bytes(self.c, 5, 3, 8),
                   wk.wushkv_weighted_workspace_bytes(self.c, 8))
        self.space = torch.full((need,), 0xFF, dtype=torch.uint8, device=gpu) if space is None else space
        self.out = [torch.empty_like(self.q, dtype=torch.float32), torch.empty_like(self.x, dtype=torch.float32),
                    torch.empty_like(self.q, dtype=torch.float32)]

    def run(self, stream=None):
        leader, shared = wk.wushkv_shared_prefixes(self.c, stream=stream)
        more = dict(workspace=self.space, stream=stream)
        wk.wushkv_prefix_attention(self.c, self.q, self.t, leader, shared, out=self.out[0], **more)
        wk.wushkv_cross_attention(self.c, self.x, self.t, self.n_tok, self.source, out=self.out[1], **more)
        wk.wushkv_weighted_attention(self.c, self.q, self.t, self.weights, out=self.out[2], **more)

    def change(self, rng):
        self.q.copy_(bf16(queries(rng, 6, 8, 128), self.q.device))
        self.source.copy_(dev_i32(rng.integers(-1, 6, 5), self.q.device))
        self.c.seq_len[:3].sub_(int(rng.integers(0, 3)))

    def same(self, other):
        return all(torch.equal(a, b) for a, b in zip((*self.out, self.weights), (*other.out, other.weights)))


def test_graphs_that_share_a_workspace(gpu):
    """Two captured runs over different caches and one workspace, replayed in turn
    with other contents, against eager ones, bit for bit."""
    one, two = Calls(gpu, 1), Calls(gpu, 2)
    a, b = Calls(gpu, 1), Calls(gpu, 2)
    b.space = a.space
    graphs, side = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], torch.cuda.Stream()
    for x in (a, b):  # (before a capture: libraries' first calls)
        x.run()
        x.weights.zero_()
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    for g, x in zip(graphs, (a, b)):
        with torch.cuda.graph(g, stream=side):
            x.run()
    torch.cuda.current_stream().wait_stream(side)
    rng = np.random.default_rng(3)
    for i in range(5):
        say("replay %d" % i)
        for x, y, g in ((one, a, graphs[0]), (two, b, graphs[1])):
            seed = int(rng.integers(1 << 30))
            x.change(np.random.default_rng(seed))
            y.change(np.random.default_rng(seed))
            x.run()
            if i % 2:
                torch.cuda.synchronize()
            g.replay()
        torch.cuda.synchronize()
        assert one.same(a) and two.same(b)


def test_other_streams_and_two_at_once(gpu):
    """Calls on streams given by hand, two caches at the same time; the default
    stream's results, bit for bit."""
    here, there = [Calls(gpu, s) for s in (4, 5)], [Calls(gpu, s) for s in (4, 5)]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for x in here:
            x.run()
        for x, side in zip(there, sides):
            x.run(stream=side)
    for side in sides:
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert here[0].same(there[0]) and here[1].same(there[1])
    # buffers made inside, on the stream
    with torch.cuda.stream(sides[0]):
        w = torch.zeros_like(here[0].weights)
        out = wk.wushkv_weighted_attention(here[0].c, here[0].q, here[0].t, w)
        cross = wk.wushkv_cross_attention(here[0].c, here[0].x, here[0].t, here[0].n_tok, here[0].source)
    torch.cuda.current_stream().wait_stream(sides[0])
    assert torch.equal(out, here[0].out[2]) and torch.equal(cross, here[0].out[1])


def test_buffers_made_for_another_stream(gpu):
    """They are none that the current stream's launches may still use: a block given
    back here goes out again on this stream alone."""
    x, side = Calls(gpu, 7), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    held = [torch.zeros(n, dtype=torch.int32, device=gpu) for n in (6, 6, 12 * 8, 6 * 8 * 128, 6 * 8 * 128)]
    held += [torch.zeros_like(x.space) for _ in range(3)]
    before = {t.data_ptr() for t in held}
    del held
    made = [*wk.wushkv_shared_prefixes(x.c, stream=side)]
    made += [wk.wushkv_weighted_attention(x.c, x.q, x.t, x.weights, stream=side)]
    made += [*wk.wushkv_evict_pages(x.c, x.pool, x.weights, dev_i32([9] * 6, gpu), max_sel=12, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert not {t.data_ptr() for t in made} & before


def test_nothing_behind_the_outputs(gpu):
    """Outputs and weights inside larger buffers: what lies round them stays."""
    x = Calls(gpu, 6)
    bufs = [torch.full((o.numel() + 512,), 7.0, device=gpu) for o in (*x.out, x.weights)]
    inner = [b[256:-256] for b in bufs]
    inner[3].zero_()
    x.out = [i.view(o.shape) for i, o in zip(inner, x.out)]
    x.weights = inner[3].view(x.weights.shape)
    want = Calls(gpu, 6)
    spaces = torch.full((x.space.numel() + 512,), 0x5A, dtype=torch.uint8, device=gpu)
    x.space = spaces[256:-256]
    x.run()
    want.run()
    torch.cuda.synchronize()
    assert x.same(want)
    for b in bufs:
        assert (b[:256] == 7).all() and (b[-256:] == 7).all()
    assert (spaces[:256] == 0x5A).all() and (spaces[-256:] == 0x5A).all()


# ------------------------------------------------------------------ large pools


def test_pages_behind_4_gib(gpu):
    """Pages at the end of a pool of more than 2^32 bytes."""
    rng = np.random.default_rng(21)
    h = Host(rng, [400, 333, 360], 8, 128, 4)
    size = h.pages.shape[2] * 8
    big = (1 << 32) // size + h.n_pages + 9
    say("a pool of %d pages of %d bytes" % (big, size))
    low = h.n_pages
    h.table = np.where(h.table >= 0, h.table + (big - low), -1).astype(np.int32)
    c = wk.WushKVCache(h.b, h.hk, h.d, h.bits, h.s_sink, h.s_keep, h.s_flush, 0.96, 0.92,
                       max_seq_len=h.s_sink + 64 * h.max_pages, win_slots=h.win_slots, page_order="none", n_pages=big, device=gpu)
    c.pages[(big - low) * size:].copy_(torch.from_numpy(h.pages.reshape(-1)))
    c.page_table.copy_(torch.from_numpy(h.table))
    c.win_k.view(torch.int16).copy_(torch.from_numpy(h.win_k.view(np.int16)))
    c.win_v.view(torch.int16).copy_(torch.from_numpy(h.win_v.view(np.int16)))
    c.seq_len.copy_(torch.from_numpy(h.seq_len))
    c.quant_end.copy_(torch.from_numpy(h.quant_end))
    q, t = queries(rng, 3, 16, 128), pages_ref.transform(rng, 8, 128)
    none = dev_i32([0, 1, 2], gpu), dev_i32([0, 0, 0], gpu)
    got = wk.wushkv_prefix_attention(c, bf16(q, gpu), f32(t, gpu), *none).cpu().numpy()
    w = torch.zeros(3, 8, h.max_pages, device=gpu)
    also = wk.wushkv_weighted_attention(c, bf16(q, gpu), f32(t, gpu), w).cpu().numpy()
    h.table = np.where(h.table >= 0, h.table - (big - low), -1).astype(np.int32)
    want, s, e = rows_exact.prefix(h, q, t, np.arange(3), np.zeros(3, int))
    assert rows_exact.off(got, want, s, e) <= 1.0 and rows_exact.off(also, want, s, e) <= 1.0


# ------------------------------------------------------------------ together


@pytest.mark.parametrize("d,bits,G,hk", [(128, 2, 4, 2), (64, 4, 8, 1)])
def test_a_serving_loop(gpu, d, bits, G, hk):
    """Forks of a prompt, the prefixes they share, attention over them, the pages'
    weights, eviction by them, attention over the lists that it gives, compaction and
    everything again: each step against its plain form."""
    say("a serving loop, d %d, %d-bit, G %d" % (d, bits, G))
    rng = np.random.default_rng([d, bits, G, 31])
    h = Host(rng, [900, 640, 333, 120, 64, 300], hk, d, bits, max_pages=16, spare=30)
    c, pool = h.cache(gpu)
    t = pages_ref.transform(rng, hk, d)
    weights = torch.zeros(h.b, hk, 16, device=gpu)
    for step, source in enumerate(([0, 1, 0, 0, -1, 1], [0, 1, 2, 2, 0, 5], [0, 1, 2, 1, 4, 5])):
        source = np.array(source)
        # a free of 4 leaves it empty; forks are of sequences that stay
        status = wk.wushkv_assign_pages(c, pool, source=dev_i32(source, gpu))
        assert np.array_equal(status.cpu().numpy(), pages_ref.assign(h, source))
        same_state(c, pool, h)
        q = queries(rng, h.b, hk * G, d)
        leader, shared = wk.wushkv_shared_prefixes(c)
        want = pages_ref.shared_prefixes(h)
        assert np.array_equal(leader.cpu().numpy(), want[0]) and np.array_equal(shared.cpu().numpy(), want[1])
        out = wk.wushkv_prefix_attention(c, bf16(q, gpu), f32(t, gpu), leader, shared)
        o, s, w = rows_exact.prefix(h, q, t, *want)
        assert rows_exact.off(out.cpu().numpy(), o, s, w) <= 1.0
        before = weights.cpu().numpy()
        same = wk.wushkv_weighted_attention(c, bf16(q, gpu), f32(t, gpu), weights)
        o, s, w, new, slack = rows_exact.weighted(h, q, t, before)
        assert rows_exact.off(same.cpu().numpy(), o, s, w) <= 1.0
        assert (np.abs(weights.cpu().numpy().astype(np.float64) - new) <= slack).all()
        x = queries(rng, 4, 2, hk * G, d)
        of = np.array([0, 4, 3, 0])
        got = wk.wushkv_cross_attention(c, bf16(x, gpu), f32(t, gpu), None, dev_i32(of, gpu))
        o, s, w = rows_exact.cross(h, x, t, None, of)
        assert rows_exact.off(got.cpu().numpy(), o, s, w) <= 1.0
        budget = np.full(h.b, 5 - step)
        at = weights.cpu().numpy()
        sel, n_sel, gone = wk.wushkv_evict_pages(c, pool, weights, dev_i32(budget, gpu), recent=2, max_sel=16)
        want = pages_ref.evict(h, at, budget, 2, 16)
        for a, b in zip((sel, n_sel, gone), want):
            assert np.array_equal(a.cpu().numpy(), b)
        same_state(c, pool, h)
        o, s, w, new, slack = rows_exact.weighted(h, q, t, np.zeros((h.b, hk, 16)), want[0], want[1])
        got = wk.wushkv_sparse_attention(c, bf16(q, gpu), f32(t, gpu), sel, n_sel)
        assert rows_exact.off(got.cpu().numpy(), o, s, w) <= 1.0
        left = torch.zeros_like(weights)
        got = wk.wushkv_weighted_attention(c, bf16(q, gpu), f32(t, gpu), left, sel, n_sel)
        assert rows_exact.off(got.cpu().numpy(), o, s, w) <= 1.0
        assert (np.abs(left.cpu().numpy().astype(np.float64) - new) <= slack).all()
        _, _, live = wk.wushkv_compact_pages(c, pool)
        assert int(live[0]) == pages_ref.compact(h)
        same_state(c, pool, h)
