"""Plain numpy forms of the page operators, in 64 bits and sequence by sequence,
written from the descriptions in include/wushkv.h, and the states the tests
give both sides."""
from __future__ import annotations

import numpy as np
import torch

import pagelayout
import paper_2609_38121_amd as wk
from workloads import synth

PAGE = 64


class Host:
    """A cache's state in host arrays: ``table``, ``pages`` uint8
    [n_pages][n_kv][page_bytes], windows as bf16 bit patterns, counters."""

    def __init__(self, rng, lens, n_kv, d, bits, s_sink=4, s_keep=32, s_flush=8, win_slots=64, spare=3, max_pages=None,
                 n_pages=None, quant=None):
        self.b, self.hk, self.d, self.bits = len(lens), n_kv, d, bits
        self.s_sink, self.s_keep, self.s_flush, self.win_slots = s_sink, s_keep, s_flush, win_slots
        self.seq_len = np.asarray(lens, np.int32)
        q = s_sink + (self.seq_len - s_keep - s_sink) // s_flush * s_flush
        self.quant_end = np.maximum(q, 0).astype(np.int32) if quant is None else np.asarray(quant, np.int32)
        need = -(-np.maximum(self.quant_end - s_sink, 0) // PAGE)
        self.max_pages = int(max(1, need.max(), max_pages or 0))
        self.n_pages = n_pages or int(need.sum()) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((self.b, self.max_pages), -1, np.int32)
        at = 0
        for i in range(self.b):
            self.table[i, :need[i]] = order[at:at + need[i]]
            at += need[i]
        self.held = need.astype(np.int32)
        self.refs = np.zeros(self.n_pages, np.int32)
        self.refs[order[:at]] = 1
        self.used = order[:at]
        self.pages = np.zeros((self.n_pages, n_kv, pagelayout.page_bytes(d, bits)), np.uint8)
        channels = np.where(rng.random(d) < 0.1, 6.0, 1.0)
        for p in self.used:
            for h in range(n_kv):
                kp = np.stack([rng.uniform(0.2, 1.5, PAGE), rng.normal(-1.0, 1.0, PAGE)], 1).astype(np.float16)
                vp = np.stack([rng.uniform(0.1, 1.0, PAGE), rng.normal(-0.5, 0.5, PAGE)], 1).astype(np.float16)
                # codes that lean one way per channel, so that boxes differ
                lean = rng.normal(0.0, 1.0, d) * np.minimum(channels, 2.0)
                top = (1 << bits) - 1
                kc = np.clip(np.round(top / 2 + lean + rng.normal(0.0, 0.6, (PAGE, d))), 0, top)
                vc = rng.integers(0, top + 1, (PAGE, d))
                self.pages[p, h] = pagelayout.encode_block(kc, vc, kp.view(np.uint16), vp.view(np.uint16), d, bits)
        self.win_k = synth.to_bf16_bits(rng.normal(0.0, 1.0, (self.b, n_kv, win_slots, d)) * channels)
        self.win_v = synth.to_bf16_bits(rng.normal(0.0, 1.0, (self.b, n_kv, d, win_slots)))

    def cache(self, dev):
        """A cache on the device with this state, and its pool."""
        c = wk.WushKVCache(self.b, self.hk, self.d, self.bits, self.s_sink, self.s_keep, self.s_flush, 0.96, 0.92,
                           max_seq_len=self.s_sink + PAGE * self.max_pages, win_slots=self.win_slots,
                           page_order="none", n_pages=self.n_pages, device=dev)
        assert c.max_pages == self.max_pages
        c.pages.copy_(torch.from_numpy(self.pages.reshape(-1)))
        c.page_table.copy_(torch.from_numpy(self.table))
        c.win_k.view(torch.int16).copy_(torch.from_numpy(self.win_k.view(np.int16)))
        c.win_v.view(torch.int16).copy_(torch.from_numpy(self.win_v.view(np.int16)))
        c.seq_len.copy_(torch.from_numpy(self.seq_len))
        c.quant_end.copy_(torch.from_numpy(self.quant_end))
        pool = wk.WushKVPool(c)
        pool.held.copy_(torch.from_numpy(self.held))
        pool.refs.copy_(torch.from_numpy(self.refs))
        return c, pool

    def end(self, b):
        return max(min(int(self.quant_end[b]), int(self.seq_len[b])), self.s_sink)

    def complete(self, b):
        return min((self.end(b) - self.s_sink) // PAGE, self.max_pages)

    def every(self, b):
        return min(-(-(self.end(b) - self.s_sink) // PAGE), self.max_pages)

    def stored(self, phys, h, values=False):
        """fp64 [64][d] keys (or values) of a page (exact: scale x code + zero)."""
        kc, vc, kp, vp = pagelayout.decode_block(self.pages[phys, h], self.d, self.bits)
        c, p = (vc, vp) if values else (kc, kp)
        p = p.view(np.float16).astype(np.float64)
        with np.errstate(invalid="ignore"):
            return c * p[:, :1] + p[:, 1:]


def transform(rng, n_kv, d):
    """fp32 [n_kv][d][d], well conditioned and not symmetric."""
    t = np.stack([synth.random_orthogonal(d, rng) * rng.uniform(0.5, 2.0, d) for _ in range(n_kv)])
    return t.astype(np.float32)


# ------------------------------------------------------------------ boxes


def box(x):
    """(codes int8 [2][d], scale fp32) of a page's stored keys x (fp64
    [64][d], rounded here to the fp32 of the stored value); every fp32 step of
    the definition is the 64-bit one rounded once (exact for one operation)."""
    f32 = np.float32
    x = x.astype(f32)
    d = x.shape[1]
    if not np.isfinite(x).all():
        return np.zeros((2, d), np.int8), f32(np.inf)
    lo, hi = x.min(0), x.max(0)
    a = max(np.abs(lo).max(), np.abs(hi).max())
    if a == 0:
        return np.zeros((2, d), np.int8), f32(0)
    s = f32(a / f32(126))
    c = np.rint(((lo + hi) * f32(0.5)) / s)
    r = np.minimum(np.ceil(np.maximum(hi - c * s, c * s - lo) / s), f32(127))
    return np.stack([c, r]).astype(np.int8), s


# ------------------------------------------------------------------ selection


def scores(host, codes, scales, q_bits, t_inv):
    """fp32 [b][hk][max_pages] (NaN where there is no complete page)."""
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(host.b, host.hk, -1, host.d)
    out = np.full((host.b, host.hk, host.max_pages), np.nan, np.float32)
    for b in range(host.b):
        for h in range(host.hk):
            rows = []
            for g in range(q.shape[2]):
                with np.errstate(invalid="ignore"):
                    qt = q[b, h, g] @ t_inv[h].astype(np.float64)
                m = np.abs(qt).max()
                if not np.isfinite(m) or m == 0:
                    rows.append((np.zeros(host.d, np.int64), 0))
                    continue
                F = int(np.clip(14 - np.frexp(m)[1], -100, 100))
                rows.append((np.clip(np.rint(qt * 2.0 ** F), -16384, 16384).astype(np.int64), F))
            for lp in range(host.complete(b)):
                p = host.table[b, lp]
                if p < 0 or p >= host.n_pages:
                    out[b, h, lp] = -np.inf
                elif np.isinf(scales[h, p]):
                    out[b, h, lp] = np.inf
                else:
                    c, r = codes[p, h].astype(np.int64)
                    out[b, h, lp] = max(np.float32(np.float32(np.float32(N @ c + np.abs(N) @ r) * scales[h, p])
                                                   * np.float32(2.0 ** -F)) for N, F in rows)
    return out


def select(host, score, top_k):
    sel = np.full((host.b, host.hk, top_k + 1), -1, np.int32)
    n = np.zeros((host.b, host.hk), np.int32)
    for b in range(host.b):
        full, every = host.complete(b), host.every(b)
        for h in range(host.hk):
            x = score[b, h, :full].astype(np.float64)
            best = np.lexsort((np.arange(full), -x))[:top_k]
            row = sorted(best) + ([full] if every > full else [])
            sel[b, h, :len(row)] = row
            n[b, h] = len(row)
    return sel, n


# ------------------------------------------------------------------ attention


def attention(host, q_bits, t_inv, sel, n_sel, sm_scale):
    """(out fp64 [b][n_q][d], bound of the kernel's error per row).

    The bound, to first order, with L the largest sum over a token of
    |q| |T^-1| |k| sm_scale (an upper bound of every partial sum of a logit):
    q~ and the logit are sums of at most d and d terms and a few rounded steps
    in fp32, q~ is taken to 24 bits (digits, or three bf16 parts): a logit is
    off by at most (2 d + 8) 2^-24 L; a weight by twice that, the exponential
    and sums of at most n tokens ((n / 64 + 80) 2^-24: a lane's own tokens, then
    trees and splits) and the 22 bits of a weight's two fp16 parts."""
    q = synth.bf16_bits_to_float(q_bits).astype(np.float64).reshape(host.b, host.hk, -1, host.d)
    G = q.shape[2]
    out = np.zeros((host.b, host.hk * G, host.d))
    tol = np.zeros((host.b, host.hk * G))
    ring = host.win_slots - host.s_sink
    for b in range(host.b):
        S, end = int(host.seq_len[b]), host.end(b)
        if S == 0:
            continue
        pos = [p for p in range(S) if p < host.s_sink or p >= end]
        slots = [p if p < host.s_sink else host.s_sink + (p - host.s_sink) % ring for p in pos]
        for h in range(host.hk):
            k = [synth.bf16_bits_to_float(host.win_k[b, h][slots]).astype(np.float64)]
            v = [synth.bf16_bits_to_float(host.win_v[b, h][:, slots]).astype(np.float64).T]
            for lp in sel[b, h, :min(max(n_sel[b, h], 0), sel.shape[2])]:
                if lp < 0 or lp >= host.max_pages or not 0 <= host.table[b, lp] < host.n_pages:
                    continue
                n = min(PAGE, end - host.s_sink - PAGE * int(lp))
                if n > 0:
                    k.append(host.stored(host.table[b, lp], h)[:n])
                    v.append(host.stored(host.table[b, lp], h, True)[:n])
            k, v = np.concatenate(k), np.concatenate(v)
            for g in range(G):
                if len(k) == 0:
                    continue
                qt = q[b, h, g] @ t_inv[h].astype(np.float64)
                x = k @ qt * sm_scale
                w = np.exp(x - x.max())
                out[b, h * G + g] = w @ v / w.sum()
                L = (np.abs(k) @ (np.abs(q[b, h, g]) @ np.abs(t_inv[h].astype(np.float64)))).max() * sm_scale
                eps = 2.0 * (2 * host.d + 8) * 2.0 ** -24 * L + (len(k) / 64 + 80) * 2.0 ** -24 + 2.0 ** -21
                tol[b, h * G + g] = 2.0 * eps * np.abs(v).max()
    return out, tol


# ------------------------------------------------------------------ assignment


def assign(host, source=None, reach=None):
    """In place on a Host; returns status.  One step after the other."""
    B = host.b
    source = np.arange(B) if source is None else np.asarray(source)
    old_table, old_q, old_s = host.table.copy(), host.quant_end.copy(), host.seq_len.copy()
    old_held = host.held.copy()
    kind = []
    for b in range(B):
        s = int(source[b])
        if s == b:
            kind.append("keep")
        elif s == -1:
            kind.append("free")
        elif 0 <= s < B and source[s] == s:
            kind.append("fork")
        else:
            kind.append("refused")
    part, filling = [0] * B, {}
    for b in range(B):
        if kind[b] in ("free", "fork"):
            for lp in range(old_held[b]):
                if 0 <= old_table[b, lp] < host.n_pages:
                    host.refs[old_table[b, lp]] -= 1
            host.table[b] = -1
            host.held[b] = host.seq_len[b] = host.quant_end[b] = 0
    for b in range(B):
        if kind[b] == "fork":
            s = int(source[b])
            q = max(min(old_q[s], old_s[s]) - host.s_sink, 0)
            n = min(q // PAGE, old_held[s])
            host.table[b, :n] = old_table[s, :n]
            for p in old_table[s, :n]:
                if 0 <= p < host.n_pages:
                    host.refs[p] += 1
            host.held[b] = n
            part[b] = int(q % PAGE != 0)
            if part[b]:
                filling[b] = (s, q // PAGE)
            host.seq_len[b], host.quant_end[b] = old_s[s], old_q[s]
            host.win_k[b], host.win_v[b] = host.win_k[s], host.win_v[s]
    free = [p for p in range(host.n_pages) if host.refs[p] <= 0]
    status = np.zeros(B, np.int32)
    for b in range(B):
        target = 0 if reach is None else min(max(-(-(int(reach[b]) - host.s_sink) // PAGE), 0), host.max_pages)
        want = max(int(host.held[b]) + part[b], target)
        missing = 0
        for lp in range(int(host.held[b]), want):
            if not free:
                host.table[b, lp] = -1
                missing += 1
                continue
            p = free.pop(0)
            host.table[b, lp] = p
            host.refs[p] = 1
            host.held[b] = lp + 1
        status[b] = -1 - missing if kind[b] == "refused" else missing
    # (a source that lacks its own page, after a call that ran out of pages,
    # gives what its row names by now)
    for b, (s, lp) in filling.items():
        if lp < host.held[b] and 0 <= host.table[s, lp] < host.n_pages:
            host.pages[host.table[b, lp]] = host.pages[host.table[s, lp]]
    return status


def compact(host, codes=None, scales=None):
    """In place on a Host (and on the boxes); returns the pages in use."""
    n = int((host.refs > 0).sum())
    holes = [p for p in range(n) if host.refs[p] <= 0]
    movers = [p for p in range(n, host.n_pages) if host.refs[p] > 0]
    to = dict(zip(movers, holes))
    for p, t in to.items():
        host.pages[t] = host.pages[p]
        host.refs[t] = host.refs[p]
        if codes is not None:
            codes[t] = codes[p]
            scales[:, t] = scales[:, p]
    host.refs[n:] = 0
    for b in range(host.b):
        for lp in range(host.max_pages):
            p = int(host.table[b, lp])
            host.table[b, lp] = to.get(p, p) if lp < host.held[b] and 0 <= p < host.n_pages else -1
    return n
