"""The attentions of many query rows in 64 bits (tests/rows_exact.py), with a tolerance
of the roundings that the kernels take, all of them independent.

u = 2^-24; sums inside a matrix instruction are taken to be off by 2 u.  Of a row's
2-norm, s is the root of the sum of the squares of

  q~      d products in fp32, 2.5 u P as in rows_exact, and a rounding by the scale (the
          30 bits of the limbs are far below): moves the output by |C|_F each.
  logits  of a page's token: sum(q~) is the first limb's (exact) and the others' sum, u;
          the start of the products is it times the middle, u, to which the first limb's
          products are added, 2 u, and the others' sum, u: s (3 |q~.(c - mid)| + 4 mid
          |sum q~|); the zero's term has its own number z + mid s, u, and sum(q~): 2
          |zero's term|; the two fused steps |zero's term - reference| + |x -
          reference|.  A reference is the whole number above a row's first largest logit
          (base 2), and moves where a page's is 8 above it or a window's is above it: it
          lies within 9 log 2 = 6.3 (windows: log 2 = 0.7) of the largest.  Of a
          window's token three parts of d terms, 3 sum_j |q~_j k_j|, and |x - reference|.
  weights the exponential 2 u and 2 u |x - reference| for its argument; in a page two
          fp16 parts of the exact product, 4 u, and 2^-25 absolute where the largest
          scale's weight is 2^5 at least: 2^-30 of the largest scale; in a window three
          bf16 parts, u.  Errors of w_t move the output by w_t (v_t - o) each.
  sums    n = 4 ceil(pages / 4) + 12 steps (four instructions a page of the wave that has
          the most, six a window unit, four waves, a division; where several workgroups
          have parts of a tile, the wave's pages are fewer by as many and more) of u of
          at most: per channel sum_t w_t s_t |c_t - middle| and sum_t w_t |v_t| of the
          windows; sum_t w_t |z_t + middle s_t|, the same in every channel; and of the
          weights' sum, |o|: sqrt(n) each.

A row may be off by 3 s, and the root mean square of the rows' errors over 1.5 s may be
1.  (rows_exact takes the steps of the last sums to err all the same way and counts them
on raw codes.)"""
import contextlib

import numpy as np

import rows_exact
from rows_exact import U


def one(host, q, T, t, sm):
    """As rows_exact.one, with w = 0."""
    d, m, nw = host.d, len(t.ks), len(t.kw)
    if m + nw == 0:
        return np.zeros(d), 0.0, 0.0, np.zeros(0), np.zeros(0)
    mid, middle = 0.5 * ((1 << host.bits) - 1), 1 << (host.bits - 1)
    k = np.concatenate([t.kc * t.ks[:, None] + t.kz[:, None], t.kw])
    v = np.concatenate([t.vc * t.vs[:, None] + t.vz[:, None], t.vw])
    qt = q @ T * sm
    x = k @ qt
    p = np.exp(x - x.max())
    w = p / p.sum()
    o = w @ v
    spread = np.linalg.norm(v - o, axis=1)
    e_q = U * (2.5 * np.sqrt((q ** 2) @ (T ** 2)).max() * sm + np.abs(qt).max())
    C = ((v - o) * w[:, None]).T @ k
    total = np.abs(qt.sum())
    zero = (t.kz + mid * t.ks) * qt.sum()
    page = np.arange(m + nw) < m
    e_x = 3.0 * (np.abs(x - x.max()) + np.where(page, 6.3, 0.7)) + np.where(page, 6.0, 3.0)
    e_x[:m] += t.ks * (3.0 * np.abs((t.kc - mid) @ qt) + 4.0 * mid * total) + 2.0 * np.abs(zero) + np.abs(zero - x.max()) + 6.3
    e_x[m:] += 3.0 * np.abs(t.kw) @ np.abs(qt)
    n = np.sqrt(4.0 * np.ceil(t.pages / 4.0) + 12.0)
    top = t.vs.max() if m else 0.0
    parts = [np.linalg.norm(C) * e_q,
             np.sqrt(((w * e_x * spread) ** 2).sum()) * U,
             np.sqrt(((t.vc - middle) ** 2).sum()) * 2.0 ** -30 * top / p.sum(),
             n * U * np.linalg.norm(w[:m] @ (t.vs[:, None] * np.abs(t.vc - middle)) + w[m:] @ np.abs(t.vw)),
             n * U * np.sqrt(d) * (w[:m] @ np.abs(t.vz + middle * t.vs)),
             n * U * np.linalg.norm(o)]
    each = U * e_x + e_q * np.abs(k).sum(1)
    return o, float(np.sqrt(np.sum(np.square(parts)))), 0.0, w, each + w @ each


@contextlib.contextmanager
def _roundings():
    was, rows_exact.one = rows_exact.one, one
    try:
        yield
    finally:
        rows_exact.one = was


def prefix(*args, **kw):
    """(out, s) of wushkv_prefix_attention."""
    with _roundings():
        return rows_exact.prefix(*args, **kw)[:2]


def cross(*args, **kw):
    """(out, s) of wushkv_cross_attention."""
    with _roundings():
        return rows_exact.cross(*args, **kw)[:2]


def weighted(*args, **kw):
    """(out, s, the pages' weights, their tolerance) of wushkv_weighted_attention."""
    with _roundings():
        out, s, _, weights, slack = rows_exact.weighted(*args, **kw)
    return out, s, weights, slack


def off(got, want, s):
    """(the largest row's error over 3 s, the rows' rms over 1.5 s); a row of no tokens
    has to be zeros."""
    e = np.linalg.norm(np.asarray(got, np.float64) - want, axis=-1)
    if (e[s == 0] != 0).any() or not (s > 0).any():
        return np.inf, np.inf
    x = e[s > 0] / s[s > 0]
    return float(x.max() / 3.0), float(np.sqrt(np.mean(x ** 2)) / 1.5)
