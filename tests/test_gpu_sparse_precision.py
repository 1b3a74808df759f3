"""The listed attention within a few roundings of its 64-bit evaluation
(sparse_exact derives how many), in states where one source of error would stand
out, split over workgroups (small batches) and a row in one workgroup each."""
import numpy as np
import pytest

import sparse_exact
from gpu_harness import say
from pages_ref import Host, transform
from test_gpu_sparse import run, some
from workloads import synth

pytestmark = pytest.mark.gpu

SHAPES = [(128, 2, 1), (128, 4, 4), (128, 2, 8), (128, 4, 8), (128, 3, 2), (64, 2, 4), (64, 4, 2), (64, 4, 8), (64, 3, 1)]


def close(gpu, h, q, t, sel, n, pick=None, what=""):
    got = run(gpu, h, q, t, sel, n)
    assert np.isfinite(got).all()
    if pick is not None:
        h, q, sel, n, got = some(h, pick), q[pick], sel[pick], n[pick], got[pick]
    want, tol = sparse_exact.rows(h, q, t, sel, n)
    most, rms = sparse_exact.off(got, want, tol)
    say("  %s: %.2e of the norm; largest %.2f, rms %.2f of what may be"
        % (what, np.linalg.norm(got - want) / np.linalg.norm(want), most, rms))
    assert most <= 1.0 and rms <= 1.0


@pytest.mark.parametrize("d,bits,G", SHAPES)
@pytest.mark.parametrize("batch", [3, 140])
def test_precision(gpu, d, bits, G, batch):
    say("d %d, %d-bit, G %d, batch %d" % (d, bits, G, batch))
    for name in sparse_exact.STATES:
        s = sparse_exact.state(name, d, bits, G, 2, batch, 64 if G != 8 else 192)
        close(gpu, *s, pick=np.arange(3), what=name)


@pytest.mark.parametrize("d,bits,G,slots", [(128, 2, 4, 64), (128, 4, 8, 128), (64, 2, 8, 64), (64, 4, 2, 192), (128, 3, 1, 64)])
@pytest.mark.parametrize("batch", [8, 150])
def test_random_lists(gpu, d, bits, G, slots, batch):
    """Sequences from nothing to several pages; lists of no page to all, with entries
    that name nothing, pages twice, counts outside the row."""
    say("lists: d %d, %d-bit, G %d, %d slots, batch %d" % (d, bits, G, slots, batch))
    rng = np.random.default_rng([d, bits, G, slots, batch])
    lens = rng.integers(0, 400, batch)
    lens[:8] = [0, 1, 4, 5, 36, 45, 100, 399]
    h = Host(rng, lens, 2, d, bits, win_slots=slots)
    q = synth.to_bf16_bits(rng.standard_normal((h.b, 2 * G, d)))
    t = transform(rng, 2, d)
    pick = np.arange(min(batch, 14))
    for width in (0, 1, 6):
        close(gpu, h, q, t, *sparse_exact.lists(rng, h, width), pick=pick, what="width %d" % width)
    sel = rng.integers(-2, 9, (h.b, 2, 40)).astype(np.int32)
    n = rng.integers(-1, 50, (h.b, 2)).astype(np.int32)
    close(gpu, h, q, t, sel, n, pick=pick, what="any entries")
    h.table[7, 1], h.table[6, 0] = h.n_pages, -9
    close(gpu, h, q, t, sel, n, pick=pick, what="pages outside the pool")


@pytest.mark.parametrize("batch,d,bits", [(2, 128, 4), (2, 64, 2), (140, 128, 2), (140, 64, 4)])
def test_large_value_scales(gpu, batch, d, bits):
    """Value scales that leave no room for lifted weights, in some pages only."""
    rng = np.random.default_rng([batch, d, bits, 1])
    h = Host(rng, [700] * 2 + [50] * (batch - 2), 2, d, bits)
    for lp, scale in ((1, 150.0), (4, 30000.0), (7, 127.0), (9, 60000.0)):
        for b in range(2):
            x = sparse_exact.params(h, h.table[b, lp], True).copy()
            x[:, :, 0] = scale
            sparse_exact.put(h, h.table[b, lp], True, x)
    q = synth.to_bf16_bits(rng.standard_normal((h.b, 4, d)))
    t = transform(rng, 2, d)
    for i in range(3):
        close(gpu, h, q, t, *sparse_exact.lists(rng, h, 10, least=4), pick=np.arange(2), what="lists %d" % i)


@pytest.mark.parametrize("s_sink,win_slots,s_keep,s_flush", [(0, 64, 32, 8), (70, 128, 32, 5), (9, 256, 180, 16), (0, 64, 0, 1),
                                                             (4, 1024, 900, 8)])
@pytest.mark.parametrize("batch,d", [(3, 128), (1, 64), (140, 128)])
def test_other_windows(gpu, s_sink, win_slots, s_keep, s_flush, batch, d):
    rng = np.random.default_rng([s_sink, win_slots, batch, d])
    lens = np.concatenate([[s_sink + s_keep + 333, s_sink + s_keep + 1, s_keep // 2], np.full(200, 20)])[:batch]
    h = Host(rng, lens, 2, d, 2, s_sink=s_sink, s_keep=s_keep, s_flush=s_flush, win_slots=win_slots, max_pages=8)
    q = synth.to_bf16_bits(rng.standard_normal((batch, 8, d)))
    t = transform(rng, 2, d)
    close(gpu, h, q, t, *sparse_exact.lists(rng, h, 5, least=2), pick=np.arange(min(batch, 3)), what="%d slots" % win_slots)


@pytest.mark.parametrize("d,bits,G", [(128, 2, 4), (128, 4, 8), (64, 2, 1)])
@pytest.mark.parametrize("batch", [3, 140])
def test_the_largest_values_in_a_window(gpu, d, bits, G, batch):
    """Finite results of values up to bf16's largest, and the other channels' as
    near as ever: the windows' sums have no room for a factor."""
    rng = np.random.default_rng([d, bits, G, batch, 4])
    h = Host(rng, [333, 90, 20] + [40] * (batch - 3), 2, d, bits)
    q = synth.to_bf16_bits(rng.standard_normal((batch, 2 * G, d)) * 0.3)
    t = transform(rng, 2, d)
    last = [p if p < 4 else 4 + (p - 4) % 60 for p in h.seq_len - 1]
    big = np.float32([3.3e38, -1e36, 5e34])
    for b in range(3):
        h.win_v[b, :, 5, last[b]] = synth.to_bf16_bits(big[b:b + 1])[0]
    sel, n = sparse_exact.lists(rng, h, 4, least=2)
    got = run(gpu, h, q, t, sel, n)[:3]
    finite = bool(np.isfinite(got).all())
    assert finite
    few = some(h, np.arange(3))
    want, _ = sparse_exact.rows(few, q[:3], t, sel[:3], n[:3])
    assert (np.abs(got[..., 5] - want[..., 5]) <= 4e-6 * np.abs(want[..., 5])).all()
    # the other channels: as if that one value were not there
    few.win_v = few.win_v.copy()
    few.win_v[:, :, 5] = 0
    want, tol = sparse_exact.rows(few, q[:3], t, sel[:3], n[:3])
    got[..., 5] = want[..., 5]
    # (weights of 2^-4 at most leave fp16 parts of 2^-21 of the largest, not 2^-33)
    room = 2.0 ** -21 * 15.0 * 2.0 * np.sqrt(64.0 * 4 * d)
    assert (np.linalg.norm(got - want, axis=-1) <= 3.0 * tol[0] + tol[1] + room).all()
