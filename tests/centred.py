"""Stored values whose sums, taken round the middle of their codes, are exact in fp32,
and round any other number are not.

Queries are zeros, so that every weight is 1.  Half of a page's tokens have a large
scale, 2^-1 (1 + i / 1024), and every code at the middle m = 2^(bits - 1); the others have
scales 2^-9 (1 + i / 1024) and any codes; every zero is -m s.  The windows' values are
zeros.  Then

  s (c - m)   of the first tokens are zeros; of the others multiples of 2^-19 below 2^-4:
              sums over up to 1000 tokens of either kind lie below 2^5 and have 24 bits;
  z + m s     are zeros;
  weights     times scales are fp16 numbers (their lo parts are zeros); every reference,
              lift and factor between two references is a power of two.

So a row's sum of values and its number of tokens are exact, however the tokens are
shared out, and its one division is rounded: off by 2^-24 of its value at most.

With codes centred on another number than m, or not at all, the first tokens add up to
more than 2^5 and are taken back by the zeros: the sums lose the others' last bits."""
import numpy as np

import pagelayout
from pages_ref import PAGE, Host


def state(rng, lens, hk, d, bits):
    h = Host(rng, lens, hk, d, bits)
    assert max(lens) <= 2000, "sums below 2^5"
    m = 1 << (bits - 1)
    for p in h.used:
        for head in range(hk):
            kc, _, kp, _ = pagelayout.decode_block(h.pages[p, head], d, bits)
            large = rng.permutation(PAGE) < PAGE // 2
            vc = np.where(large[:, None], m, rng.integers(0, 1 << bits, (PAGE, d)))
            s = (1.0 + rng.integers(0, 1024, PAGE) / 1024.0) * np.where(large, 2.0 ** -1, 2.0 ** -9)
            vp = np.stack([s, -m * s], 1).astype(np.float16)
            assert np.array_equal(vp.astype(np.float64)[:, 0], s) and np.array_equal(vp.astype(np.float64)[:, 1], -m * s)
            h.pages[p, head] = pagelayout.encode_block(kc, vc, kp, vp.view(np.uint16), d, bits)
    h.win_v[:] = 0
    return h


def values(h, b, head, pages):
    """Codes [n][d], scales and zeros [n] of the tokens in these (sequence, page)s."""
    c, s, z = [], [], []
    for seq, lp in pages:
        n = min(PAGE, h.end(seq) - h.s_sink - PAGE * lp)
        _, vc, _, vp = pagelayout.decode_block(h.pages[h.table[seq, lp], head], h.d, h.bits)
        c.append(vc[:n])
        s.append(vp.view(np.float16).astype(np.float64)[:n, 0])
        z.append(vp.view(np.float16).astype(np.float64)[:n, 1])
    return np.concatenate(c).astype(np.float64), np.concatenate(s), np.concatenate(z)


def row(h, b, head, pages=None):
    """The output of a row that attends to these pages (sequence b's own, by default)
    and to b's windows: fp64 [d]."""
    pages = [(b, i) for i in range(h.every(b))] if pages is None else pages
    live = int(h.seq_len[b]) - max(h.end(b) - h.s_sink, 0)  # of the windows
    c, s, z = values(h, b, head, pages)
    return (s[:, None] * c + z[:, None]).sum(0) / (len(s) + live)


def fp32_row(h, b, head, middle):
    """The same with fp32 sums of s (c - middle), 32 tokens at a time, and of z + middle s,
    four waves' pages apart, as the attentions of many rows add them up."""
    f32 = np.float32
    pages = h.every(b)
    live = int(h.seq_len[b]) - max(h.end(b) - h.s_sink, 0)
    total, n = np.zeros(h.d, f32), live
    for w in range(4):
        acc, zero = np.zeros(h.d, f32), np.zeros(16, f32)
        for lp in range(w, pages, 4):
            c, s, z = values(h, b, head, [(b, lp)])
            n += len(s)
            for i in range(0, len(s), 32):
                acc = (acc + (s[i:i + 32, None] * (c[i:i + 32] - middle)).sum(0)).astype(f32)
            for i, x in enumerate((z + middle * s).astype(f32)):
                zero[i // 4] += x
        total = (total + (acc + zero.sum(dtype=f32))).astype(f32)
    return total / f32(n)


def off(got, want):
    """The largest error over 2^-24 of the value (a value of zero is one)."""
    e = np.abs(np.asarray(got, np.float64) - want)
    if (e[want == 0] != 0).any():
        return np.inf
    return float((e[want != 0] / np.abs(want[want != 0])).max() * 2.0 ** 24)
