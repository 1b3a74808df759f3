"""Attention over stored sequences that several queries share, attention that
adds up what each page received, and the pages that leave by it.

Each case is one call (``run``) of one operator over the range a serving loop
meets:

  prefixes  which sequences start with the same pages, from the page table
  prefix    a decode query per sequence; pages that sequences share at their
            start are attended to once for all of them
  cross     queries of other sequences, of any length, over stored states (no
            mask; several query sequences may share one stored sequence)
  weighted  decode attention over all or listed pages that adds every page's
            attention weight to what it received before
  evict     the pages with the least weight leave their sequences

``run`` computes them in elementary torch operations, or, where ``own`` is
true, through the framework's entry points on the same tensors.  ``exact`` is
the definition in 64 bits.  Shapes follow the repository's workloads: sink of
4, 128 recent tokens, flushes of 8, keys with eight outlier channels x10.
"""
import math

import numpy as np
import torch

own = False

SINK, KEEP, FLUSH, SLOTS, PAGE = 4, 128, 8, 192, 64


def _case(op, **over):
    c = dict(op=op, batch=1, members=1, n_kv=8, group=4, d=128, bits=2, lo=1, hi=1, own_lo=140, own_hi=140, tok=1,
             ragged=False, top_k=0, recent=2)
    c.update(over)
    return c


def listed():
    """name, then what it stands for."""
    return [
        # eight answers sampled from one short prompt
        _case("prefixes", name="prefixes 8 forks", members=8, lo=700, hi=700, own_lo=140, own_hi=300),
        # four documents, sixteen questions about each, the forks of different depth
        _case("prefixes", name="prefixes 4 x 16 of 8K-32K", batch=4, members=16, lo=8192, hi=32768, own_lo=140, own_hi=900,
              ragged=True),
        # the smallest call: two sequences, small heads
        _case("prefix", name="prefix 2 on a short prompt", members=2, n_kv=1, d=64, lo=500, hi=500, own_lo=150, own_hi=200),
        # eight prompts sampled eight ways, eight query heads per kv head, 4-bit codes
        _case("prefix", name="prefix 8 x 8 on 5K-8K G8 4-bit", batch=8, members=8, group=8, bits=4, lo=5000, hi=8192,
              own_lo=140, own_hi=1000, ragged=True),
        # the large serving batch behind one long document
        _case("prefix", name="prefix 64 on 32K", members=64, lo=32768, hi=32768, own_lo=140, own_hi=600),
        # the smallest call: one generated token, small heads
        _case("cross", name="cross one token, 700 states", n_kv=2, group=1, d=64, lo=700, hi=700),
        # four hypotheses of each of sixteen inputs
        _case("cross", name="cross 16 x 4 tokens, 4-bit", batch=16, members=4, bits=4, lo=2000, hi=8192),
        # eight prompts of up to 256 tokens over the states of their inputs
        _case("cross", name="cross 8 x 256 tokens", batch=8, lo=1000, hi=3000, tok=256, ragged=True),
        # the smallest attention that keeps count, over everything
        _case("weighted", name="weighted one short sequence", n_kv=1, d=64, lo=700, hi=700),
        # the large serving batch, each sequence down to 64 pages
        _case("weighted", name="weighted 64 x 16K-32K", batch=64, lo=16384, hi=32768, top_k=64),
        # a small batch, a page or two over its budget each
        _case("evict", name="evict 8 short sequences", batch=8, n_kv=1, lo=600, hi=2000, top_k=6),
        # the large serving batch, after its prompts
        _case("evict", name="evict 64 x 16K-32K", batch=64, lo=16384, hi=32768, top_k=64, recent=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prefixes", "prefix", "prefix", "prefix", "cross", "cross", "cross", "weighted", "weighted", "evict"])
    shape = dict(n_kv=rng.choice([1, 2, 4, 8]), group=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 128]),
                 bits=rng.choice([2, 2, 3, 4]), ragged=rng.choice([False, True]))
    if op in ("prefixes", "prefix"):
        members = _log(rng, 2, 64)
        batch = _log(rng, 1, 64 // members)
        hi = _log(rng, 200, min(32768, 8000000 // (batch * members * shape["group"]), 65536 // batch))
        own_hi = _log(rng, 140, 2000)
        return _case(op, batch=batch, members=members, lo=max(100, int(hi * rng.uniform(0.3, 1.0))), hi=hi, own_lo=130,
                     own_hi=own_hi, **shape)
    if op == "cross":
        batch = _log(rng, 1, 16)
        members = rng.choice([1, 1, 2, 4, 5])
        hi = _log(rng, 1, min(8192, 32768 // batch))
        rows = batch * members * shape["group"]
        tok = _log(rng, 1, max(1, min(512, 8192 // rows, 24000000 // (rows * hi))))
        return _case(op, batch=batch, members=members, lo=max(1, int(hi * rng.uniform(0.2, 1.0))), hi=hi, tok=tok, **shape)
    batch = _log(rng, 1, 64)
    if op == "weighted":
        hi = _log(rng, 100, min(65536, 200000 // batch))
        top_k = rng.choice([0, _log(rng, 1, max(1, min(hi // PAGE, 4096 // batch)))])
    else:
        hi = _log(rng, 300, 32768)
        top_k = _log(rng, 1, hi // PAGE)
    return _case(op, batch=batch, lo=max(1, int(hi * rng.uniform(0.2, 1.0))), hi=hi, top_k=top_k, recent=rng.choice([0, 1, 5]),
                 **shape)


# ------------------------------------------------------------------ sizes


def _store(bits):
    return 4 if bits == 3 else bits


def _page_bytes(c):
    return PAGE * (2 * c["d"] * _store(c["bits"]) // 8 + 8)


def _spread(hi, lo, n):
    return np.round(np.linspace(hi, lo, n)).astype(np.int64) if n > 1 else np.array([hi])


def _sharing(c):
    return c["op"] in ("prefixes", "prefix")


def _batch(c):
    """Stored sequences."""
    return c["batch"] * c["members"] if _sharing(c) else c["batch"]


def _forks(c):
    """(leader, pages that the sequence has in common with it): sequence b is
    member b // groups of group b % groups, whose first member leads."""
    n, b = c["batch"], np.arange(_batch(c))
    pages = np.maximum(1, (_spread(c["hi"], c["lo"], n) - SINK) // PAGE)[b % n]
    short = (b // n % 4 == 3) & c["ragged"]
    return b % n, np.where(short, np.maximum(1, pages - pages // 4), pages)


def _lengths(c):
    """The sequences' lengths (from the case: the work does not depend on the seed)."""
    if _sharing(c):
        b = np.arange(_batch(c))
        return SINK + PAGE * _forks(c)[1] + c["own_lo"] + b * 7919 % (c["own_hi"] - c["own_lo"] + 1)
    return _spread(c["hi"], c["lo"], c["batch"])


def _quant_end(s):
    return np.maximum(0, SINK + (s - KEEP - SINK) // FLUSH * FLUSH)


def _pages_of(q):
    """Complete pages, and pages in all, of the quantised positions [SINK, q)."""
    n = np.maximum(q - SINK, 0)
    return n // PAGE, -(-n // PAGE)


def _max_pages(c):
    return max(1, -(-max(0, int(_lengths(c).max()) - SINK) // PAGE))


def _common(c):
    """Pages at the start of each row that are another sequence's too, and
    whose they are."""
    b = np.arange(_batch(c))
    full, every = _pages_of(_quant_end(_lengths(c)))
    if _sharing(c):
        lead, n = _forks(c)
        return np.where(b == lead, 0, n), lead
    if c["op"] == "evict":  # every other sequence is a fork of the one before
        lead = b - b % 2
        return np.where(b == lead, 0, np.minimum(full, full[lead]) // 2), lead
    return np.zeros_like(b), b


def _own_pages(c):
    return _pages_of(_quant_end(_lengths(c)))[1] - _common(c)[0]


def _pool_pages(c):
    """Physical pages of the pool."""
    pages = _pages_of(_quant_end(_lengths(c)))[1] if c["op"] == "prefixes" else _own_pages(c)
    return int(pages.sum() * 1.1) + 1


def _tokens(c):
    """cross: the query sequences' token counts."""
    n = c["batch"] * c["members"]
    if not c["ragged"]:
        return np.full(n, c["tok"])
    return np.maximum(1, c["tok"] - np.arange(n) * 37 % (c["tok"] * 2 // 3 + 1))


def _selected(c):
    """weighted: pages of each list."""
    full, every = _pages_of(_quant_end(_lengths(c)))
    return every if c["top_k"] == 0 else np.minimum(full, c["top_k"]) + (every - full)


def work(case):
    c = case
    d, hk, g, b, mp = c["d"], c["n_kv"], c["group"], _batch(c), _max_pages(c)
    s = _lengths(c)
    q = _quant_end(s)
    full, every = _pages_of(q)
    window = int((s - np.maximum(q - SINK, 0)).sum()) * hk
    if c["op"] == "prefixes":
        return {"bytes": 4.0 * int(full.sum()) + 16 * b, "flops": 0}
    if c["op"] == "evict":
        left = np.minimum(full, c["top_k"]) + (every - full)
        return {"bytes": 4.0 * hk * int(full.sum()) + 8.0 * int(every.sum()) + 8.0 * _pool_pages(c) + 4.0 * hk * int(left.sum())
                + 24.0 * b, "flops": 0}
    rows = b * hk * g
    pages = int(_own_pages(c).sum()) * hk
    seen = int((s.astype(np.int64)).sum()) * hk
    extra = 0.0
    if c["op"] == "cross":
        tok = _tokens(c)
        rows = int(tok.sum()) * hk * g
        seen = int((tok * s[np.arange(len(tok)) // c["members"]]).sum()) * hk
    if c["op"] == "weighted":
        pages = int(_selected(c).sum()) * hk
        seen = pages * PAGE + window
        extra = 8.0 * pages + (4.0 * pages if c["top_k"] else 0.0)
    return {"bytes": pages * (_page_bytes(c) + 4.0 / hk) + window * d * 4 + hk * d * d * 4 + rows * d * 6 + extra,
            "flops": 2.0 * rows * d * d + 4.0 * g * d * seen}


# ------------------------------------------------------------------ inputs


def _gen(seed, *tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence([seed, *tag]).generate_state(1, np.uint64)[0] >> 1))
    return g


def _word_maps(d, sb):
    """For every word and element of a code region: (token, channel) and the
    bit, of keys and of values (the page layout of the cache)."""
    span = 32 // sb
    e = np.arange(span)
    L, t, w = np.meshgrid(np.arange(d // 2), np.arange(4), np.arange(sb), indexing="ij")
    k = sb * t + w
    at = ((k // 4) * 2 * d + 4 * L + k % 4).ravel()
    kt = np.empty((at.size, span), np.int64)
    kc = np.empty_like(kt)
    kt[at] = (4 * (L % 16) + t).ravel()[:, None]
    kc[at] = (32 * (L // 16) + span * w).ravel()[:, None] + e
    kbit = 2 * sb * (e % (span // 2)) + sb * (e // (span // 2))
    nw = d * sb // 128
    L, c, u = np.meshgrid(np.arange(64), np.arange(2), np.arange(2 * nw), indexing="ij")
    k = c * 2 * nw + u
    at = ((k // 4) * 256 + 4 * L + k % 4).ravel()
    vt = np.empty((at.size, span), np.int64)
    vc = np.empty_like(vt)
    vt[at] = (32 * c + 8 * (L // 16)).ravel()[:, None] + e % 8
    vc[at] = (16 * (u * (span // 8)) + L % 16).ravel()[:, None] + 16 * (e // 8)
    field = np.array([6, 10, 8, 12, 2, 0, 4, 14] if sb == 2 else [4, 0, 8, 12])
    vbit = 16 * (e % 2) + field[4 * (e // 8) + (e % 8) // 2]
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return [(dev(kt), dev(kc), dev(kbit)), (dev(vt), dev(vc), dev(vbit))]


def _pack(x, bits, maps):
    """Page blocks (bytes) of [n][2][64][d] keys and values: every token's
    codes evenly spaced between its least and its largest entry."""
    n, d = x.shape[0], x.shape[-1]
    lo = x.amin(-1, keepdim=True)
    zero = lo.half()
    scale = ((x.amax(-1, keepdim=True) - lo) / (2 ** bits - 1)).half()
    code = ((x - zero.float()) / scale.float()).round_().clamp_(0, 2 ** bits - 1).to(torch.int32)
    parts = []
    for i, (t, c, bit) in enumerate(maps):
        words = (code[:, i][:, t, c] << bit.to(torch.int32)).sum(-1, dtype=torch.int32)
        parts.append(words.view(torch.uint8).reshape(n, -1))
    for i in range(2):
        parts.append(torch.stack([scale[:, i, :, 0], zero[:, i, :, 0]], -1).contiguous().view(torch.uint8).reshape(n, -1))
    return torch.cat(parts, 1)


class _State:
    """The tensors of a cache and of one call."""


def _tables(c, r):
    """Page table (physical pages in random order), and references."""
    b, mp, n = _batch(c), _max_pages(c), _pool_pages(c)
    full, every = _pages_of(_quant_end(_lengths(c)))
    common, lead = _common(c)
    if c["op"] == "prefixes":  # half of the forks left their leader earlier
        common = np.where(r.random(b) < 0.5, np.ceil(common * r.random(b)).astype(np.int64), common)
    mine = every - common
    first = np.cumsum(mine) - mine
    free = r.permutation(n)
    lp = np.arange(mp)
    table = np.full((b, mp), -1, np.int64)
    for i in range(b):  # (a sequence's leader comes before it)
        table[i, :common[i]] = table[lead[i], :common[i]]
        table[i, common[i]:every[i]] = free[first[i]:first[i] + mine[i]]
    if c["op"] == "evict":  # pages that left before
        table[(r.random((b, mp)) < 0.1) & (lp < full[:, None])] = -1
    refs = np.bincount(table[table >= 0], minlength=n)
    return table, refs


def prepare(case, seed):
    c, dev = case, "cuda"
    b, hk, d, n, mp = _batch(c), c["n_kv"], c["d"], _pool_pages(c), _max_pages(c)
    r = np.random.default_rng([seed, 1])
    st = _State()
    st.case = c
    st.cache = None
    whole = c["op"] not in ("prefixes", "evict")  # (those read no page)
    if own:
        import paper_2609_38121_amd as wk
        st.wk = wk
        st.cache = wk.WushKVCache(b, hk, d, c["bits"], SINK, KEEP, FLUSH, 0.96, 0.92, max_seq_len=int(_lengths(c).max()),
                                  win_slots=SLOTS, page_order="none", n_pages=n)
        for name in ("page_table", "win_k", "win_v", "seq_len", "quant_end"):
            setattr(st, name, getattr(st.cache, name))
        n = st.cache.n_pages
        st.pages = st.cache.pages.view(n, hk, -1)
        st.pool = wk.WushKVPool(st.cache)
        st.refs, st.held = st.pool.refs, st.pool.held
    else:
        st.pages = torch.zeros(n if whole else 1, hk, _page_bytes(c), dtype=torch.uint8, device=dev)
        st.page_table = torch.full((b, mp), -1, dtype=torch.int32, device=dev)
        st.win_k = torch.zeros(b, hk, SLOTS, d, dtype=torch.bfloat16, device=dev)
        st.win_v = torch.zeros(b, hk, d, SLOTS, dtype=torch.bfloat16, device=dev)
        st.seq_len, st.quant_end, st.held = (torch.zeros(b, dtype=torch.int32, device=dev) for _ in range(3))
        st.refs = torch.zeros(n, dtype=torch.int32, device=dev)

    s = _lengths(c)
    full, every = _pages_of(_quant_end(s))
    put = lambda t, a: t.copy_(torch.from_numpy(np.ascontiguousarray(a)))  # noqa: E731
    new = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(dev)  # noqa: E731
    table, refs = _tables(c, r)
    # (the sequences in any order, where that is what the call has to find out)
    order = r.permutation(b) if c["op"] == "prefixes" else np.arange(b)
    put(st.seq_len, s[order])
    put(st.quant_end, _quant_end(s)[order])
    put(st.page_table, table[order])
    put(st.refs, refs)
    put(st.held, every[order])

    outlier = torch.ones(d, device=dev)
    outlier[torch.from_numpy(r.choice(d, 8, replace=False)).to(dev)] = 10.0
    if whole:
        maps = _word_maps(d, _store(c["bits"]))
        common = _common(c)[0]
        for i in range(b):  # a sequence's own pages at a time: keys that drift from page to page, values that do not
            m = int(every[i] - common[i])
            if not m:
                continue
            g = _gen(seed, 2, i)
            x = torch.randn(m * hk, 2, PAGE, d, generator=g, device=dev)
            x[:, 0] = (x[:, 0] + 0.7 * torch.randn(m * hk, 1, d, generator=g, device=dev)) * outlier
            at = torch.from_numpy(table[i, common[i]:every[i]]).to(dev)
            st.pages[at] = _pack(x, c["bits"], maps).view(m, hk, -1)
        g = _gen(seed, 3)
        st.win_k.copy_(torch.randn(st.win_k.shape, generator=g, device=dev) * outlier)
        st.win_v.copy_(torch.randn(st.win_v.shape, generator=g, device=dev))
        a = r.standard_normal((hk, d, d))
        u, _ = np.linalg.qr(a)
        scale = np.exp(r.uniform(math.log(0.5), math.log(2.0), (hk, 1, d)))
        st.t_inv = torch.from_numpy(((u * scale) @ np.swapaxes(u, 1, 2)).astype(np.float32)).to(dev)
        shape = (b, hk * c["group"], d)
        if c["op"] == "cross":
            shape = (b * c["members"], c["tok"], hk * c["group"], d)
        st.q = torch.randn(shape, generator=_gen(seed, 4), device=dev).to(torch.bfloat16)
    if c["op"] == "prefix":
        lead, n = _forks(c)
        st.leader, st.shared = new(lead), new(np.where(lead == np.arange(b), 0, n))
    if c["op"] == "cross":
        st.source, st.n_tok = new(np.arange(b * c["members"]) // c["members"]), new(_tokens(c))
    if c["op"] in ("weighted", "evict"):
        # a few pages receive most of the weight; some never any
        w = torch.randn(b, hk, mp, generator=_gen(seed, 5), device=dev).mul_(2.0).exp_()
        never = torch.rand(b, 1, mp, generator=_gen(seed, 6), device=dev) < 0.1
        st.weights = torch.where(never, torch.zeros_like(w), w).contiguous()
    st.sel = st.n_sel = None
    if c["op"] == "weighted" and c["top_k"]:
        # a list per sequence and kv head: distinct complete pages in ascending order, then the page that is being filled
        width = c["top_k"] + 1
        sel = np.full((b, hk, width), -1)
        for i in range(b):
            k = min(int(full[i]), c["top_k"])
            for h in range(hk):
                sel[i, h, :k] = np.sort(r.choice(int(full[i]), k, replace=False)) if k else []
            if every[i] > full[i]:
                sel[i, :, k] = full[i]
        st.sel, st.n_sel = new(sel), new(np.repeat(_selected(c)[:, None], hk, 1))
    if c["op"] == "evict":
        st.budget = new(np.where(np.arange(b) % 8 == 7, -1, c["top_k"]))
    if own:
        # buffers that a serving loop keeps
        space = lambda n: torch.empty(n, dtype=torch.uint8, device=dev)  # noqa: E731
        if c["op"] == "prefixes":
            st.leader, st.shared = torch.empty_like(st.seq_len), torch.empty_like(st.seq_len)
        if whole:
            st.out = torch.empty(st.q.shape, device=dev)
        if c["op"] == "prefix":
            st.space = space(wk.wushkv_prefix_workspace_bytes(st.cache, hk * c["group"]))
        if c["op"] == "cross":
            st.space = space(wk.wushkv_cross_workspace_bytes(st.cache, b * c["members"], c["tok"], hk * c["group"]))
        if c["op"] == "weighted":
            st.space = space(wk.wushkv_weighted_workspace_bytes(st.cache, hk * c["group"], c["top_k"] + 1 if c["top_k"] else mp))
        if c["op"] == "evict":
            st.table, st.refs2 = torch.empty_like(st.page_table), torch.empty_like(st.refs)
            st.sel, st.n_sel = new(np.zeros((b, hk, mp))), new(np.zeros((b, hk)))
            st.evicted = torch.empty_like(st.seq_len)
    return st


# ------------------------------------------------------------------ the plain forms


def _places(d, sb):
    """(token, channel) -> word and bit in a code region, keys then values."""
    span = 32 // sb
    t, ch = torch.meshgrid(torch.arange(PAGE), torch.arange(d), indexing="ij")
    rest = ch % 32 % span
    k = sb * (t % 4) + ch % 32 // span
    key = (k // 4) * 2 * d + 4 * (16 * (ch // 32) + t // 4) + k % 4
    kbit = 2 * sb * (rest % (span // 2)) + sb * (rest // (span // 2))
    per = span // 8
    nt = ch // 16
    k = (t // 32) * (d * sb // 64) + nt // per
    val = (k // 4) * 256 + 4 * (16 * (t // 8 % 4) + ch % 16) + k % 4
    field = torch.tensor([6, 10, 8, 12, 2, 0, 4, 14] if sb == 2 else [4, 0, 8, 12])
    vbit = 16 * (t % 2) + field[4 * (nt % per) + t % 8 // 2]
    return [x.to("cuda", torch.int32) for x in (key, kbit, val, vbit)]


def _stored(blocks, d, bits, values):
    """fp32 [..., 64, d] keys (or values) of page blocks [..., page_bytes]:
    scale x code + zero, rounded once (the sum is exact in 64 bits)."""
    sb = _store(bits)
    key, kbit, val, vbit = _places(d, sb)
    region = 8 * d * sb
    at, bit = (val, vbit) if values else (key, kbit)
    first = region if values else 0
    words = blocks[..., first:first + region].contiguous().view(torch.int32)
    codes = (words[..., at] >> bit) & (2 ** sb - 1)
    first = 2 * region + (4 * PAGE if values else 0)
    par = blocks[..., first:first + 4 * PAGE].contiguous().view(torch.float16).unflatten(-1, (PAGE, 2))
    if values:
        return codes.float() * par[..., :1].float() + par[..., 1:].float()
    return (codes.double() * par[..., :1].double() + par[..., 1:].double()).float()


def _counts(st):
    """Complete pages, and pages in all, of the sequences."""
    end = torch.maximum(torch.minimum(st.quant_end, st.seq_len) - SINK, torch.zeros_like(st.seq_len))
    return end // PAGE, (end + PAGE - 1) // PAGE


def _gathered(st, phys):
    """Keys and values, fp32 [rows][n_kv][tokens][d], of the pages phys [rows][pages]."""
    c = st.case
    blocks = st.pages[torch.clamp(phys, min=0).long()].transpose(1, 2)
    return [_stored(blocks, c["d"], c["bits"], v).flatten(2, 3) for v in (False, True)]


def _live(st, lp, phys):
    """Which of the tokens [rows][pages][64] of logical pages lp count."""
    end = torch.maximum(torch.minimum(st.quant_end, st.seq_len), torch.full_like(st.seq_len, SINK))
    token = SINK + PAGE * lp[..., None] + torch.arange(PAGE, device="cuda")
    return (phys >= 0)[..., None] & (token < end[:, None, None])


def _window_live(st):
    """The windows' slots [batch][slots] that hold positions: the sink's, and
    the ring's from the oldest position on."""
    end = torch.maximum(torch.minimum(st.quant_end, st.seq_len), torch.full_like(st.seq_len, SINK))
    slot = torch.arange(SLOTS, device="cuda")
    turn = torch.remainder(slot - SINK - (end - SINK)[:, None], SLOTS - SINK)
    return torch.where(slot < SINK, slot < st.seq_len[:, None], turn < (st.seq_len - end).clamp(min=0)[:, None])


def _windows(st):
    return st.win_k.float(), st.win_v.float().transpose(2, 3)


def _logits(st, rows, keys, mask):
    x = torch.matmul(rows, keys.transpose(2, 3)) * (1.0 / math.sqrt(st.case["d"]))
    return torch.where(mask, x, torch.full_like(x, -math.inf))


def _entries(st, lp):
    """Physical pages of logical ones [batch][..], -1 where there is none."""
    mp = st.page_table.shape[1]
    phys = st.page_table.gather(1, torch.clamp(lp, 0, mp - 1).flatten(1).long()).view(lp.shape)
    return torch.where((lp >= 0) & (lp < mp), phys, -1)


def _prefixes(st):
    full, _ = _counts(st)
    t = st.page_table
    b, mp = t.shape
    lp = torch.arange(mp, device="cuda")
    same = (t[:, None] == t[None]) & (lp < torch.minimum(full[:, None], full)[..., None])
    same = torch.cumprod(same.int(), -1) * (t >= 0)
    common = torch.where(same > 0, lp.int() + 1, 0).amax(-1)
    at = torch.arange(b, device="cuda")
    common = torch.where(at[:, None] == at, 0, common)
    best = common.amax(1)
    mate = (common >= best[:, None]) | (at[:, None] == at)
    leader = torch.where(best > 0, torch.where(mate, at, b).amin(1), at)
    return {"leader": leader.int(), "shared": torch.where(leader == at, 0, best).int()}


def _prefix(st):
    c = st.case
    n, m, hk, g, d = c["batch"], c["members"], c["n_kv"], c["group"], c["d"]
    b = n * m
    at = torch.arange(b, device="cuda")
    _, every = _counts(st)
    # the leaders attend to what any of their sequences shares
    lead = st.leader.long()
    shared = torch.where(lead == at, torch.zeros_like(st.shared).index_reduce(0, lead, st.shared, "amax"), st.shared)
    q = torch.matmul(st.q.float().view(b, hk, g, d), st.t_inv)
    # sequences of a group side by side: b = member x groups + group
    group = lambda x: x.view(m, n, *x.shape[1:]).transpose(0, 1)  # noqa: E731
    rows = group(q).transpose(1, 2).reshape(n, hk, m * g, d)
    most = int(_forks(c)[1].max())
    keys, values = _gathered(st, st.page_table[:n, :most])
    seen = torch.arange(most * PAGE, device="cuda") < PAGE * group(shared)[:, :, None]  # [groups][members][tokens]
    near = _logits(st, rows, keys, seen[:, None, :, None].expand(n, 1, m, g, -1).reshape(n, 1, m * g, -1))
    # each sequence's own pages and windows
    width = int((_pages_of(_quant_end(_lengths(c)))[1] - _forks(c)[1]).max())
    lp = shared[:, None] + torch.arange(width, device="cuda")
    lp = torch.where(lp < every[:, None], lp, -1)
    phys = _entries(st, lp)
    k2, v2 = [torch.cat(x, 2) for x in zip(_gathered(st, phys), _windows(st))]
    mask = torch.cat([_live(st, lp, phys).flatten(1), _window_live(st)], 1)
    far = _logits(st, q, k2, mask[:, None, None])
    alone = lambda x: x.view(n, hk, m, g, -1).permute(2, 0, 1, 3, 4).reshape(b, hk, g, -1)  # noqa: E731
    top = torch.maximum(alone(near.amax(-1, keepdim=True)), far.amax(-1, keepdim=True))
    near = torch.exp(near - group(top).transpose(1, 2).reshape(n, hk, m * g, 1))
    far = torch.exp(far - top)
    total = alone(near.sum(-1, keepdim=True)) + far.sum(-1, keepdim=True)
    return ((alone(torch.matmul(near, values)) + torch.matmul(far, v2)) / total).reshape(b, hk * g, d)


def _cross(st):
    c = st.case
    b, m, tok, hk, g, d = c["batch"], c["members"], c["tok"], c["n_kv"], c["group"], c["d"]
    _, every = _counts(st)
    lp = torch.arange(st.page_table.shape[1], device="cuda").expand(b, -1)
    phys = torch.where(lp < every[:, None], st.page_table, -1)
    keys, values = [torch.cat(x, 2) for x in zip(_gathered(st, phys), _windows(st))]
    mask = torch.cat([_live(st, lp, phys).flatten(1), _window_live(st)], 1)
    # (query sequences of one stored sequence are side by side)
    rows = st.q.float().view(b, m * tok, hk, g, d).permute(0, 2, 1, 3, 4)
    rows = torch.matmul(rows.reshape(b, hk, m * tok * g, d), st.t_inv)
    x = _logits(st, rows, keys, mask[:, None, None])
    p = torch.exp(x - x.amax(-1, keepdim=True))
    out = torch.matmul(p, values) / p.sum(-1, keepdim=True)
    out = out.view(b, hk, m * tok, g, d).transpose(1, 2).reshape(b * m, tok, hk * g, d)
    there = torch.arange(tok, device="cuda") < st.n_tok[:, None]
    return torch.where(there[:, :, None, None], out, torch.zeros_like(out))


def _weighted(st):
    c = st.case
    b, hk, g, d = c["batch"], c["n_kv"], c["group"], c["d"]
    mp = st.page_table.shape[1]
    _, every = _counts(st)
    sel, n_sel = st.sel, st.n_sel
    if sel is None:
        sel = torch.arange(mp, dtype=torch.int32, device="cuda").expand(b, hk, mp)
        n_sel = every[:, None].expand(b, hk)
    lp = torch.where(torch.arange(sel.shape[2], device="cuda") < n_sel[..., None], sel, -1)
    phys = _entries(st, lp)
    blocks = st.pages[torch.clamp(phys, min=0).long(), torch.arange(hk, device="cuda")[:, None]]
    keys, values = [torch.cat([_stored(blocks, d, c["bits"], v).flatten(2, 3), w], 2)
                    for v, w in zip((False, True), _windows(st))]
    mask = torch.cat([_live(st, lp.flatten(1), phys.flatten(1)).view(b, hk, -1),
                      _window_live(st)[:, None].expand(b, hk, -1)], 2)
    q = torch.matmul(st.q.float().view(b, hk, g, d), st.t_inv)
    x = _logits(st, q, keys, mask[:, :, None])
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    mass = p[..., :-SLOTS].unflatten(-1, (-1, PAGE)).sum(-1).sum(2)
    st.weights.scatter_add_(2, torch.clamp(lp, min=0).long(), torch.where(phys >= 0, mass, 0.0))
    return {"out": torch.matmul(p, values).view(b, hk * g, d), "weights": st.weights}


def _evict(st):
    c = st.case
    b, mp = st.page_table.shape
    hk = c["n_kv"]
    full, every = _counts(st)
    lp = torch.arange(mp, device="cuda")
    there = (st.page_table >= 0) & (lp < st.held[:, None])
    live = there & (lp < full[:, None])
    free = live & (lp < (full - c["recent"])[:, None])
    over = torch.minimum((live.sum(1) - st.budget).clamp(min=0), free.sum(1))
    over = torch.where(st.budget < 0, torch.zeros_like(over), over)
    score = st.weights.double().sum(1).float()
    # the candidates by weight, the lowest page first among equals
    order = torch.sort(torch.where(free, score, math.inf), dim=1, stable=True)[1]
    order = order.gather(1, torch.sort((~free.gather(1, order)).int(), dim=1, stable=True)[1])
    gone = torch.zeros_like(free).scatter(1, order, lp < over[:, None])
    table = torch.where(gone, -1, st.page_table)
    n = st.refs.numel()
    left = torch.where(gone, st.page_table, n).flatten().long()
    refs = torch.nn.functional.pad(st.refs, (0, 1)).index_add(0, left, torch.full_like(left, -1, dtype=torch.int32))[:n]
    kept = (there & (lp < every[:, None]) & ~gone)
    sel = torch.sort(torch.where(kept, lp, mp), dim=1)[0]
    sel = torch.where(sel < mp, sel, -1).int()[:, None].expand(b, hk, mp).contiguous()
    n_sel = kept.sum(1, dtype=torch.int32)[:, None].expand(b, hk).contiguous()
    return {"table": table, "refs": refs, "sel": sel, "n_sel": n_sel, "evicted": over.int()}


def run(st):
    c = st.case
    if own:
        wk = st.wk
        if c["op"] == "prefixes":
            wk.wushkv_shared_prefixes(st.cache, leader=st.leader, shared=st.shared)
            return {"leader": st.leader, "shared": st.shared}
        if c["op"] == "prefix":
            return wk.wushkv_prefix_attention(st.cache, st.q, st.t_inv, st.leader, st.shared, out=st.out, workspace=st.space)
        if c["op"] == "cross":
            return wk.wushkv_cross_attention(st.cache, st.q, st.t_inv, n_tok=st.n_tok, source=st.source, out=st.out,
                                             workspace=st.space)
        if c["op"] == "weighted":
            wk.wushkv_weighted_attention(st.cache, st.q, st.t_inv, st.weights, sel=st.sel, n_sel=st.n_sel, out=st.out,
                                         workspace=st.space)
            return {"out": st.out, "weights": st.weights}
        wk.wushkv_evict_pages(st.cache, st.pool, st.weights, st.budget, recent=c["recent"], sel=st.sel, n_sel=st.n_sel,
                              table_out=st.table, refs_out=st.refs2, evicted=st.evicted)
        return {"table": st.table, "refs": st.refs2, "sel": st.sel, "n_sel": st.n_sel, "evicted": st.evicted}
    return {"prefixes": _prefixes, "prefix": _prefix, "cross": _cross, "weighted": _weighted, "evict": _evict}[c["op"]](st)


# ------------------------------------------------------------------ in 64 bits


def _read(blocks, d, bits, values, maps):
    """fp64 [n][64][d] of page blocks [n][page_bytes], word by word."""
    sb = _store(bits)
    region = 8 * d * sb
    t, ch, bit = maps[1 if values else 0]
    w = blocks[:, region * values:region * (1 + values)].contiguous().view(torch.int32).long() & 0xFFFFFFFF
    out = torch.zeros(blocks.shape[0], PAGE, d, dtype=torch.float64, device="cuda")
    out[:, t, ch] = ((w[:, :, None] >> bit) & (2 ** sb - 1)).double()
    first = 2 * region + 4 * PAGE * values
    par = blocks[:, first:first + 4 * PAGE].contiguous().view(torch.float16).view(-1, PAGE, 2).double()
    return out * par[:, :, :1] + par[:, :, 1:]

def _window(c, st, b, h, s, start):
    """fp64 keys and values of the positions in sequence b's windows."""
    pos = np.concatenate([np.arange(min(SINK, s)), np.arange(start, s)])
    slots = torch.from_numpy(np.where(pos < SINK, pos, SINK + (pos - SINK) % (SLOTS - SINK))).cuda()
    return st.win_k[b, h, slots].double(), st.win_v[b, h][:, slots].double().t()


def exact(case, seed):
    c = case
    if c["op"] in ("prefixes", "evict"):
        return None  # whole numbers
    st = prepare(case, seed)
    d, hk, g = c["d"], c["n_kv"], c["group"]
    maps = _word_maps(d, _store(c["bits"]))
    s, q = _lengths(c), _quant_end(_lengths(c))
    full, every = _pages_of(q)
    table = st.page_table.cpu().numpy()
    out = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    soft = lambda rows, k, v: torch.softmax(rows @ k.t() / math.sqrt(d), -1) @ v  # noqa: E731

    def paged(b, h, pages):
        """Keys and values of sequence b's listed logical pages, and of its windows."""
        start = max(int(min(q[b], s[b])), SINK)
        k, v = [], []
        if len(pages):
            blocks = st.pages[torch.from_numpy(table[b, pages].astype(np.int64)).cuda(), h]
            n = torch.from_numpy(np.minimum(PAGE, start - SINK - PAGE * np.asarray(pages))).cuda()
            here = (torch.arange(PAGE, device="cuda") < n[:, None]).flatten()
            k.append(_read(blocks, d, c["bits"], False, maps).flatten(0, 1)[here])
            v.append(_read(blocks, d, c["bits"], True, maps).flatten(0, 1)[here])
        kw, vw = _window(c, st, b, h, int(s[b]), start)
        return torch.cat(k + [kw]), torch.cat(v + [vw])

    if c["op"] == "cross":
        tok, m = _tokens(c), c["members"]
        for b in range(c["batch"]):
            for h in range(hk):
                k, v = paged(b, h, np.arange(every[b]))
                for i in range(b * m, b * m + m):
                    rows = st.q[i, :tok[i], h * g:(h + 1) * g].double() @ st.t_inv[h].double()
                    out[i, :tok[i], h * g:(h + 1) * g] = soft(rows.flatten(0, 1), k, v).view(int(tok[i]), g, d)
        return out
    if c["op"] == "prefix":
        lead, n = _forks(c)
        for first in range(c["batch"]):
            for h in range(hk):
                for b in range(first, _batch(c), c["batch"]):
                    if b == first:  # the leader's pages, read once for its sequences
                        k0, v0 = paged(b, h, np.arange(n[b]))
                        k0, v0 = k0[:PAGE * n[b]], v0[:PAGE * n[b]]
                    k, v = paged(b, h, np.arange(n[b], every[b]))
                    rows = st.q[b, h * g:(h + 1) * g].double() @ st.t_inv[h].double()
                    out[b, h * g:(h + 1) * g] = soft(rows, torch.cat([k0[:PAGE * n[b]], k]), torch.cat([v0[:PAGE * n[b]], v]))
        return out
    weights = st.weights.double()
    for b in range(c["batch"]):
        for h in range(hk):
            pages = np.arange(every[b])
            if st.sel is not None:
                pages = st.sel[b, h, :int(st.n_sel[b, h])].cpu().numpy().astype(np.int64)
            k, v = paged(b, h, pages)
            rows = st.q[b, h * g:(h + 1) * g].double() @ st.t_inv[h].double()
            p = torch.softmax(rows @ k.t() / math.sqrt(d), -1)
            out[b, h * g:(h + 1) * g] = p @ v
            start = max(int(min(q[b], s[b])), SINK)
            sums = torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), p.sum(0).cumsum(0)])
            ends = torch.from_numpy(np.cumsum(np.minimum(PAGE, start - SINK - PAGE * pages))).cuda()
            if len(pages):
                each = sums[ends] - sums[torch.cat([ends.new_zeros(1), ends[:-1]])]
                weights[b, h, torch.from_numpy(pages).cuda()] += each
    return {"out": out, "weights": weights}
