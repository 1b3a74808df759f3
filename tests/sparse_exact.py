"""The attention over listed pages in 64 bits with a tolerance near what fp32
arithmetic gives, states in which one source of error would stand out, and the
same evaluation with a mistake planted in it.

The tolerance, of a row's 2-norm, is made of independent roundings (a rounding
is off by u = 2^-24 of its value at most; sums inside a matrix instruction are
taken to be off by a unit, 2 u):

  q~      d products summed in fp32, in runs of 16 and a tree of 8, or 32 steps of
          the matrix instruction: with partial sums of sqrt(i / d) P, P = sqrt(sum_i
          q_i^2 T_ij^2), either is off by 2.5 u P (rms) at most; then a rounding by the
          scale and one to 24 bits of the largest entry.  An error e of q~ (per
          channel) moves the output by |C|_F e, C = sum_t w_t (v_t - o) k_t^T.
  logits  of a page's token: the exact digit sums are combined, scaled and added to
          the zero's term: at most 4 u (|s q~.(c - mid)| + |(z + mid s) sum q~|); of a
          window's, sums of d terms, u sum_j |q~_j k_j|; and 2 u |x - max x| for the
          exponent's argument.
  weights the exponential 2 u; in a page the product with the value scale u and two
          fp16 parts 4 u (relative; and 2^-25 absolute where the largest weight is
          2^lift, lift 8, or 0 with a value scale of 128 or more); in a window three
          bf16 parts u.  Errors of w_t, of logit or weight, move the output by w_t (v_t - o) each.
  sums    over the tokens in fp32, of sum_t w_t s_t c_t, of sum_t w_t |z_t| and of the
          windows' sum_t w_t |v_t|, per channel: two instructions a page of the wave
          that has the most, each off by a unit of half of the sum (and always the
          same way, should it truncate), and four steps after them: u (2 ceil(pages /
          4) + 4), whole.

What is independent (all but the last) is s, the last is w: a row may be off by 3 s +
w, and the root mean square of the rows' errors over 1.5 s + w may be 1."""
import numpy as np

import pagelayout
from pages_ref import PAGE, Host, transform
from workloads import synth

U = 2.0 ** -24


def bf16(x):
    return synth.bf16_bits_to_float(synth.to_bf16_bits(x)).astype(np.float64)


def rows(host, q_bits, t_inv, sel, n_sel, plant=None, scale=None):
    """(out fp64 [b][n_q][d], s and w [2][b][n_q]).  plant: None, or a mistake: "last
    page" left out, "two parts" (windows), "short sums" (19 bits), "no lift", "not
    centred"; s and w are those of the true evaluation."""
    f32 = np.float32
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(host.b, host.hk, -1, host.d)
    G, d = q.shape[2], host.d
    sm = 1.0 / np.sqrt(d) if scale is None else scale
    mid = 0.5 * ((1 << host.bits) - 1)
    out, tol = np.zeros((host.b, host.hk * G, d)), np.zeros((2, host.b, host.hk * G))
    ring = host.win_slots - host.s_sink
    rng = np.random.default_rng(1)
    for b in range(host.b):
        S, end = int(host.seq_len[b]), host.end(b)
        pos = [p for p in range(S) if p < host.s_sink or p >= end]
        slots = [p if p < host.s_sink else host.s_sink + (p - host.s_sink) % ring for p in pos]
        for h in range(host.hk):
            kw = synth.bf16_bits_to_float(host.win_k[b, h][slots]).astype(np.float64)
            vw = synth.bf16_bits_to_float(host.win_v[b, h][:, slots]).astype(np.float64).T
            kc, ks, kz, vc, vs, vz = [np.zeros((0, d))], [[]], [[]], [np.zeros((0, d))], [[]], [[]]
            pages = 0
            listed = [int(p) for p in sel[b, h, :min(max(n_sel[b, h], 0), sel.shape[2])]]
            listed = [p for p in listed if 0 <= p < host.max_pages and 0 <= host.table[b, p] < host.n_pages
                      and end - host.s_sink - PAGE * p > 0]
            for lp in listed:
                n = min(PAGE, end - host.s_sink - PAGE * lp)
                a, c, e, f = pagelayout.decode_block(host.pages[host.table[b, lp], h], d, host.bits)
                e, f = (x.view(np.float16).astype(np.float64)[:n] for x in (e, f))
                for x, y in ((kc, a[:n]), (ks, e[:, 0]), (kz, e[:, 1]), (vc, c[:n]), (vs, f[:, 0]), (vz, f[:, 1])):
                    x.append(y)
                pages += 1
            kc, ks, kz, vc, vs, vz = (np.concatenate(x).astype(np.float64) for x in (kc, ks, kz, vc, vs, vz))
            m, nw = len(ks), len(kw)
            if m + nw == 0:
                continue
            k = np.concatenate([kc * ks[:, None] + kz[:, None], kw])
            v = np.concatenate([vc * vs[:, None] + vz[:, None], vw])
            T = t_inv[h].astype(np.float64)
            for g in range(G):
                qt = q[b, h, g] @ T * sm
                x = k @ qt
                p = np.exp(x - x.max())
                w = p / p.sum()
                o = w @ v
                out[b, h * G + g] = o
                # ---- the tolerance
                spread = np.linalg.norm(v - o, axis=1)
                P = np.sqrt((q[b, h, g] ** 2) @ (T ** 2)).max() * sm
                e_q = U * (2.5 * P + np.abs(qt).max())
                C = ((v - o) * w[:, None]).T @ k
                e_x = 2.0 * np.abs(x - x.max()) + np.where(np.arange(m + nw) < m, 7.0, 3.0)
                e_x[:m] += 4.0 * (np.abs(ks * ((kc - mid) @ qt)) + np.abs((kz + mid * ks) * qt.sum()))
                e_x[m:] += np.abs(kw) @ np.abs(qt)
                big = (vs >= 128).any() if m else False
                floor = 2.0 ** -25 * (1.0 if big else 2.0 ** -8) / p.sum()
                sums = w[:m] @ (vs[:, None] * vc) + w[:m] @ np.abs(vz) + w[m:] @ np.abs(vw)
                parts = [np.linalg.norm(C) * e_q,
                         np.sqrt(((w * e_x * spread) ** 2).sum()) * U,
                         np.sqrt((vc ** 2).sum()) * floor]
                tol[:, b, h * G + g] = (np.sqrt(np.sum(np.square(parts))),
                                        U * (2.0 * np.ceil(pages / 4.0) + 4.0) * np.linalg.norm(sums))
                # ---- a planted mistake
                if plant is None:
                    continue
                if plant == "last page":
                    if m:
                        w = w.copy()
                        w[m - min(PAGE, end - host.s_sink - PAGE * listed[-1]):m] = 0.0
                        out[b, h * G + g] = w @ v / w.sum()
                elif plant == "two parts":
                    hi = bf16(qt)
                    y = x.copy()
                    y[m:] = kw @ (hi + bf16(qt - hi))
                    z = np.exp(y - x.max())
                    hi = bf16(z[m:])
                    zz = z.copy()
                    zz[m:] = hi + bf16(z[m:] - hi)
                    out[b, h * G + g] = zz @ v / z.sum()
                elif plant == "short sums":
                    acc = np.zeros(d)
                    for i in range(0, m, 32):
                        acc = acc + (w[i:min(i + 32, m)] * vs[i:i + 32][:min(32, m - i)]) @ vc[i:i + 32]
                        acc *= 1.0 + 2.0 ** -19 * rng.uniform(-0.5, 0.5, d)
                    out[b, h * G + g] = acc + w[:m] @ vz + w[m:] @ vw
                elif plant == "no lift":
                    ps = p[:m] * vs
                    hi = ps.astype(np.float16).astype(np.float64)
                    lo = (ps - hi).astype(np.float16).astype(np.float64)
                    out[b, h * G + g] = ((hi + lo) @ vc + p[:m] @ vz + p[m:] @ vw) / p.sum()
                else:
                    assert plant == "not centred"
                    y = x.copy()
                    a = (ks.astype(f32) * (kc @ qt).astype(f32)).astype(f32)
                    y[:m] = (a + (kz.astype(f32) * f32(qt.sum())).astype(f32)).astype(f32)
                    z = np.exp(y - x.max())
                    out[b, h * G + g] = z @ v / z.sum()
    return out, tol


def off(got, want, tol):
    """(the largest row's error over 3 s + w, the rows' rms over 1.5 s + w; a row of
    zeros has to be one)."""
    e = np.linalg.norm(np.asarray(got, np.float64) - want, axis=-1)
    if not (e[tol[0] == 0] == 0).all() or not (tol[0] > 0).any():
        return np.inf, np.inf
    e, (s, w) = e[tol[0] > 0], tol[:, tol[0] > 0]
    return float((e / (3.0 * s + w)).max()), float(np.sqrt(np.mean((e / (1.5 * s + w)) ** 2)))


def lists(rng, host, width, least=0):
    """Random pages in random order, least to width of them where there are as many."""
    sel = np.full((host.b, host.hk, width), -1, np.int32)
    n = np.zeros((host.b, host.hk), np.int32)
    for b in range(host.b):
        for h in range(host.hk):
            most = min(width, host.every(b))
            n[b, h] = rng.integers(min(least, most), most + 1)
            sel[b, h, :n[b, h]] = rng.permutation(host.every(b))[:n[b, h]]
    return sel, n


def params(host, page, values):
    """View [n_kv][64][2] of a page's scales and zeros."""
    par = host.pages.shape[2] - (256 if values else 512)
    return host.pages[page, :, par:par + 256].view(np.float16).reshape(host.hk, PAGE, 2)


def put(host, page, values, x):
    par = host.pages.shape[2] - (256 if values else 512)
    host.pages[page, :, par:par + 256] = np.ascontiguousarray(x.astype(np.float16)).reshape(host.hk, 128).view(np.uint8)


STATES = {"pages": "last page", "windows": "two parts", "sums": "short sums", "peak": "no lift", "far zeros": "not centred"}


def state(name, d, bits, G, hk, batch, win_slots=64):
    """(host, q, T^-1, sel, n_sel) of a state; STATES names the mistake that it shows.
    Sequences after the third are short."""
    rng = np.random.default_rng([len(name), d, bits, G, hk, batch, win_slots])
    keep = 32 if win_slots == 64 else win_slots - 20
    lens = [700 + keep, 333 + keep, 500 + keep] if name != "windows" else [6, 14, 9]
    lens = lens[:batch] + [50] * max(0, batch - 3)
    h = Host(rng, lens, hk, d, bits, s_keep=keep, win_slots=win_slots)
    q = rng.standard_normal((batch, hk * G, d))
    t = transform(rng, hk, d)
    sel, n = lists(rng, h, 9, least=5)
    if name == "windows":   # a few tokens there, logits about one
        n[:] = 0
        q *= 0.2
    if name == "sums":      # every token about as heavy: the sums over them are the result
        q *= 0.05
    if name == "peak":      # one token far above the others, small value scales
        q = np.abs(q) * 0.02
        t = np.repeat(np.eye(d, dtype=np.float32)[None], hk, 0)
        for p in h.used:
            x = params(h, p, False).copy()
            x[:, :, 1] = -x[:, :, 0] * 0.5 * ((1 << bits) - 1)
            put(h, p, False, x)
            x = params(h, p, True).copy()
            x[:, :, 0], x[:, :, 1] = 2.0 ** -6, 0.0
            put(h, p, True, x)
        for b in range(min(batch, 3)):
            for head in range(hk):
                p = h.table[b, sel[b, head, 0]]
                x = params(h, p, False).copy()
                x[head, 3, 1] += 8.0 * np.sqrt(d) / np.abs(synth.bf16_bits_to_float(synth.to_bf16_bits(q[b, head * G]))).sum()
                put(h, p, False, x)
        h.win_v[:] = 0
        q[:] = q[:, [i // G * G for i in range(hk * G)]]  # (the group's heads alike)
    if name == "far zeros":  # key codes round the middle, queries of one sign
        q = 4.0 + 0.1 * q
        t = np.repeat(np.eye(d, dtype=np.float32)[None], hk, 0)
        for p in h.used:
            for head in range(hk):
                _, vc, kp, vp = pagelayout.decode_block(h.pages[p, head], d, bits)
                kc = rng.integers((1 << bits) // 2 - 1, (1 << bits) // 2 + 1, (PAGE, d))
                x = kp.view(np.float16).astype(np.float64)
                x[:, 1] = -x[:, 0] * 0.5 * ((1 << bits) - 1) + rng.normal(0.0, 0.01, PAGE)
                h.pages[p, head] = pagelayout.encode_block(kc, vc, x.astype(np.float16).view(np.uint16), vp, d, bits)
        h.win_k = synth.to_bf16_bits(synth.bf16_bits_to_float(h.win_k) * 0.1)
    return h, synth.to_bf16_bits(q), t, sel, n
