"""The attentions of many query rows (prefix, cross, weighted) in 64 bits, row by
row, with a tolerance near what fp32 arithmetic gives.

A row is (its q~, the stored tokens that it attends to).  The tolerance, of a row's
2-norm, is made of independent roundings (one is off by u = 2^-24 of its value at
most; sums inside a matrix instruction are taken to be off by a unit, 2 u):

  q~      d products summed in fp32 in 32 steps of the matrix instruction, two
          chains: off by 2.5 u P at most, P = sqrt(sum_i q_i^2 T_ij^2); a rounding
          by the scale and one to 24 bits of the largest entry.  An error e of q~
          moves the output by |C|_F e, C = sum_t w_t (v_t - o) k_t^T.
  logits  of a page's token: six limbs, each added onto the sum before it, 12 u of
          the centred product and of sum(q~) in the zero's term; the start of the
          sum, u s mid |sum q~|; the two fused steps, u (|zero's term - reference| +
          |x - reference|), references within 12 of a row's maximum.  Of a window's
          token three parts of d terms, 3 u sum_j |q~_j k_j|.
  weights the exponential 2 u and 2 u |x - reference| for its argument; in a page
          two fp16 parts of the exact product 4 u (and 2^-25 absolute where the
          largest weight is at least 2^4 / 8: value scales lie up to eight times
          above the one that their power of two goes by); in a window three bf16
          parts u.  Errors of w_t move the output by w_t (v_t - o) each.
  sums    over the tokens in fp32, of sum_t w_t s_t c_t, of sum_t w_t |z_t| and of
          sum_t w_t |v_t| (windows), per channel: four instructions a page of the
          wave that has the most, six a window unit, and the references' moves and
          merges, each off by a unit of half of the sum: u (4 ceil(pages / 4) + 24),
          whole.

What is independent (all but the last) is s, the last is w: a row may be off by 3 s
+ w."""
import numpy as np

import pagelayout
from pages_ref import PAGE
from workloads import synth

U = 2.0 ** -24


class Tokens:
    """Stored tokens: codes, scales and zeros of pages' tokens, then the windows'."""

    def __init__(self, host, b, h, pages, windows=True):
        """Of sequence b: ``pages``, (sequence, logical page) each; its windows."""
        d = host.d
        kc, ks, kz, vc, vs, vz = [np.zeros((0, d))], [[]], [[]], [np.zeros((0, d))], [[]], [[]]
        self.pages, self.first = 0, []
        for s, lp in pages:
            n = min(PAGE, host.end(s) - host.s_sink - PAGE * lp) if 0 <= lp < host.max_pages else 0
            ok = n > 0 and 0 <= host.table[s, lp] < host.n_pages
            self.first.append(sum(len(x) for x in ks))
            if not ok:
                continue
            a, c, e, f = pagelayout.decode_block(host.pages[host.table[s, lp], h], d, host.bits)
            e, f = (x.view(np.float16).astype(np.float64)[:n] for x in (e, f))
            for x, y in ((kc, a[:n]), (ks, e[:, 0]), (kz, e[:, 1]), (vc, c[:n]), (vs, f[:, 0]), (vz, f[:, 1])):
                x.append(y)
            self.pages += 1
        self.kc, self.ks, self.kz, self.vc, self.vs, self.vz = (np.concatenate(x).astype(np.float64)
                                                                for x in (kc, ks, kz, vc, vs, vz))
        self.first.append(len(self.ks))
        S, end = int(host.seq_len[b]), host.end(b)
        pos = [p for p in range(S) if p < host.s_sink or p >= end] if windows else []
        ring = host.win_slots - host.s_sink
        slots = [p if p < host.s_sink else host.s_sink + (p - host.s_sink) % ring for p in pos]
        self.kw = synth.bf16_bits_to_float(host.win_k[b, h][slots]).astype(np.float64).reshape(-1, d)
        self.vw = synth.bf16_bits_to_float(host.win_v[b, h][:, slots]).astype(np.float64).T.reshape(-1, d)


def one(host, q, T, t, sm):
    """(output, s, w, the tokens' weights and the most that each may be off, of its
    value) of a row: q fp64 [d], T fp64 [d][d]."""
    d, m, nw = host.d, len(t.ks), len(t.kw)
    if m + nw == 0:
        return np.zeros(d), 0.0, 0.0, np.zeros(0), np.zeros(0)
    mid = 0.5 * ((1 << host.bits) - 1)
    k = np.concatenate([t.kc * t.ks[:, None] + t.kz[:, None], t.kw])
    v = np.concatenate([t.vc * t.vs[:, None] + t.vz[:, None], t.vw])
    qt = q @ T * sm
    x = k @ qt
    p = np.exp(x - x.max())
    w = p / p.sum()
    o = w @ v
    spread = np.linalg.norm(v - o, axis=1)
    P = np.sqrt((q ** 2) @ (T ** 2)).max() * sm
    e_q = U * (2.5 * P + np.abs(qt).max())
    C = ((v - o) * w[:, None]).T @ k
    away = np.abs(x - x.max()) + 12.0
    e_x = 3.0 * away + np.where(np.arange(m + nw) < m, 7.0, 3.0)
    total = np.abs(qt.sum())
    zero = np.abs(t.kz + mid * t.ks) * total
    e_x[:m] += 12.0 * np.abs(t.ks * ((t.kc - mid) @ qt)) + 13.0 * zero + t.ks * mid * total + np.abs(x.max())
    e_x[m:] += 3.0 * np.abs(t.kw) @ np.abs(qt)
    sums = w[:m] @ (t.vs[:, None] * t.vc) + w[:m] @ np.abs(t.vz) + w[m:] @ np.abs(t.vw)
    top = t.vs.max() if m else 0.0
    parts = [np.linalg.norm(C) * e_q, np.sqrt(((w * e_x * spread) ** 2).sum()) * U,
             np.sqrt((t.vc ** 2).sum()) * 2.0 ** -25 * top / (2.0 * p.sum())]
    each = U * e_x + e_q * np.abs(k).sum(1)
    return (o, float(np.sqrt(np.sum(np.square(parts)))), U * (4.0 * np.ceil(t.pages / 4.0) + 24.0) * np.linalg.norm(sums), w,
            each + w @ each)


def off(got, want, s, w):
    """The largest row's error over 3 s + w (a row of no tokens has neither and has
    to be zeros; one of a single token has w alone: its sums p v and p, each rounded)."""
    e = np.linalg.norm(np.asarray(got, np.float64) - want, axis=-1)
    none = s + w == 0
    if not (e[none] == 0).all():
        return np.inf
    return float((e[~none] / (3.0 * s + w)[~none]).max()) if (~none).any() else 0.0


def prefix(host, q_bits, t_inv, leader, shared, scale=None):
    """(out [b][n_q][d], s, w [b][n_q]) of wushkv_prefix_attention."""
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(host.b, host.hk, -1, host.d)
    G, sm = q.shape[2], 1.0 / np.sqrt(host.d) if scale is None else scale
    out, tol = np.zeros((host.b, host.hk * G, host.d)), np.zeros((2, host.b, host.hk * G))
    for b in range(host.b):
        if host.seq_len[b] == 0:
            continue
        le, s = int(leader[b]), 0
        if 0 <= le < host.b and le != b:
            s = max(min(int(shared[b]), host.complete(b), host.complete(le)), 0)
        pages = [(le if i < s else b, i) for i in range(host.every(b))]
        for h in range(host.hk):
            t = Tokens(host, b, h, pages)
            for g in range(G):
                o, e, w, _, _ = one(host, q[b, h, g], t_inv[h].astype(np.float64), t, sm)
                out[b, h * G + g], tol[:, b, h * G + g] = o, (e, w)
    return out, tol[0], tol[1]


def cross(host, q_bits, t_inv, n_tok, source, scale=None):
    """(out [n][max_tok][n_q][d], s, w) of wushkv_cross_attention."""
    n, tok = q_bits.shape[:2]
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(n, tok, host.hk, -1, host.d)
    G, sm = q.shape[3], 1.0 / np.sqrt(host.d) if scale is None else scale
    out, tol = np.zeros((n, tok, host.hk * G, host.d)), np.zeros((2, n, tok, host.hk * G))
    for i in range(n):
        b = i if source is None else int(source[i])
        m = tok if n_tok is None else min(max(int(n_tok[i]), 0), tok)
        if not 0 <= b < host.b or host.seq_len[b] == 0 or m == 0:
            continue
        for h in range(host.hk):
            t = Tokens(host, b, h, [(b, p) for p in range(host.every(b))])
            for k in range(m):
                for g in range(G):
                    o, e, w, _, _ = one(host, q[i, k, h, g], t_inv[h].astype(np.float64), t, sm)
                    out[i, k, h * G + g], tol[:, i, k, h * G + g] = o, (e, w)
    return out, tol[0], tol[1]


def weighted(host, q_bits, t_inv, weights, sel=None, n_sel=None, scale=None):
    """(out, s, w) of wushkv_weighted_attention, and the weights in fp64 and their
    tolerance: a page's is the sum of its tokens', each off by its logit's and
    exponential's error and by their mean, the row's; then fp32 sums over the
    tokens, the heads and onto what was there, u each."""
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(host.b, host.hk, -1, host.d)
    G, sm = q.shape[2], 1.0 / np.sqrt(host.d) if scale is None else scale
    out, tol = np.zeros((host.b, host.hk * G, host.d)), np.zeros((2, host.b, host.hk * G))
    new, slack = weights.astype(np.float64), np.zeros(weights.shape)
    for b in range(host.b):
        if host.seq_len[b] == 0:
            continue
        for h in range(host.hk):
            pages = list(range(host.every(b))) if sel is None else \
                [int(p) for p in sel[b, h, :min(max(n_sel[b, h], 0), sel.shape[2])]]
            t = Tokens(host, b, h, [(b, p) for p in pages])
            T = t_inv[h].astype(np.float64)
            for g in range(G):
                o, e, w, p, each = one(host, q[b, h, g], T, t, sm)
                out[b, h * G + g], tol[:, b, h * G + g] = o, (e, w)
                for i, lp in enumerate(pages):
                    a, z = t.first[i], t.first[i + 1]
                    if z > a:
                        new[b, h, lp] += p[a:z].sum()
                        slack[b, h, lp] += (p[a:z] * each[a:z]).sum() + 24.0 * U * p[a:z].sum()
    return out, tol[0], tol[1], new, slack + G * U * np.abs(new)
