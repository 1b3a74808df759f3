"""WUSH-KV online hot path for AMD Instinct MI355X (gfx950).

Python binding over the C ABI in include/wushkv.h.  The functions here have
the names of the C entry points and only marshal arguments; PyTorch supplies
device memory and the current HIP stream.

    cache = WushKVCache(batch=8, n_kv_heads=8, head_dim=128, bits=2,
                        s_sink=4, s_keep=128, s_flush=8,
                        kappa_k=0.96, kappa_v=0.92, max_seq_len=8192)
    wushkv_append(cache, k_new, v_new, n_new, t_k)
    out = wushkv_decode_attention(cache, q, t_k_inv)
"""
from __future__ import annotations

import ctypes
import math
import operator

from . import _lib
from ._lib import (BoundsDesc, CacheDesc, PoolDesc, WushKVError, PAGE_TOKENS, check, header_functions,
                   status_string)

__all__ = [
    "WushKVCache", "WushKVError", "wushkv_append", "wushkv_decode_attention",
    "wushkv_decode_attention_noalloc", "wushkv_decode_step",
    "wushkv_decode_workspace_bytes", "wushkv_dequant", "wushkv_page_bytes",
    "wushkv_status_string", "wushkv_abi_version", "wushkv_timing_enable",
    "wushkv_timing_read", "wushkv_timing_launches", "wushkv_quest_alpha", "wushkv_wush_transform", "wushkv_read_probe",
    "WushKVBounds", "WushKVPool", "wushkv_page_bounds", "wushkv_select_pages",
    "wushkv_select_workspace_bytes", "wushkv_sparse_attention", "wushkv_sparse_workspace_bytes",
    "wushkv_assign_pages", "wushkv_compact_pages", "wushkv_compact_workspace_bytes",
    "wushkv_shared_prefixes", "wushkv_prefix_attention", "wushkv_prefix_workspace_bytes", "wushkv_cross_attention",
    "wushkv_cross_workspace_bytes", "wushkv_weighted_attention", "wushkv_weighted_workspace_bytes", "wushkv_evict_pages",
    "PAGE_TOKENS",
    "header_functions",
]


def _torch():
    import torch
    return torch


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream_handle(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    # the current stream's handle without a Stream object (2.8 us a call, as
    # much as a kernel launch)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def wushkv_page_bytes(head_dim: int, bits: int) -> int:
    return _lib.lib().wushkv_page_bytes(head_dim, bits)


def wushkv_status_string(status: int) -> str:
    return status_string(status)


def wushkv_abi_version() -> int:
    return _lib.lib().wushkv_abi_version()


def wushkv_quest_alpha(bits: int) -> float:
    """The Gaussian-MSE-optimal clip multiplier alpha_b of Eq. (5)."""
    return _lib.lib().wushkv_quest_alpha(bits)


def wushkv_timing_enable(slots: int) -> None:
    check(_lib.lib().wushkv_timing_enable(slots), "wushkv_timing_enable")


def wushkv_timing_read(name_substr: str = ""):
    """(launch count, summed milliseconds per launch) of recorded launches
    whose kernel name contains name_substr; reading does not clear the
    record (re-enabling does)."""
    cnt = ctypes.c_int32()
    ms = ctypes.c_double()
    check(_lib.lib().wushkv_timing_read(name_substr.encode(), ctypes.byref(cnt),
                                        ctypes.byref(ms)), "wushkv_timing_read")
    return cnt.value, ms.value


def wushkv_timing_launches():
    """[(kernel name, milliseconds)] of every launch recorded since timing
    was enabled, in launch order."""
    L = _lib.lib()
    out = []
    name = ctypes.c_char_p()
    ms = ctypes.c_double()
    for i in range(L.wushkv_timing_count()):
        check(L.wushkv_timing_launch(i, ctypes.byref(name), ctypes.byref(ms)), "wushkv_timing_launch")
        out.append((name.value.decode(), ms.value))
    return out


class _Described:
    """Device arrays and the C descriptor that names them.  A program may put
    another contiguous tensor of the same type, shape and device in an array's
    place: the descriptor follows it (a captured graph keeps the old one)."""

    def __setattr__(self, name, value):
        desc = self.__dict__.get("_desc")
        if desc is not None and name in _FIELDS[type(desc)]:
            old = self.__dict__[name]
            if not isinstance(value, _torch().Tensor) or value.device != old.device:
                raise ValueError("%s must be a tensor on %s" % (name, old.device))
            setattr(desc, name, _check(old.get_device(), value, name, old.dtype, old.shape))
        object.__setattr__(self, name, value)


# the arrays of each descriptor
_FIELDS = {d: frozenset(n for n, t in d._fields_ if t is ctypes.c_void_p) for d in (CacheDesc, BoundsDesc, PoolDesc)}


class WushKVCache(_Described):
    """Device memory of one WUSH-KV cache plus its C descriptor.

    Allocates (torch, on ``device``): the page pool, the page table, the bf16
    windows, the per-sequence counters and the append's arrival counts, all
    zero-initialised except the windows, which may hold anything (they are
    only read where live).
    ``page_order`` "linear" maps logical page i of sequence b to physical
    page b * max_pages + i; "random" draws a seeded permutation of a pool
    ``pool_factor`` times the needed size, "none" leaves the table empty (-1)
    for wushkv_assign_pages to fill from a pool of ``n_pages`` pages (by
    default as many as the other orders take).  ``codec`` is "pclip" (Eq. (7),
    clip quantiles kappa_k / kappa_v) or "quest" (Eq. (5), clip multiplier
    ``quest_alpha``, by default the library's wushkv_quest_alpha(bits)).
    """

    def __init__(self, batch, n_kv_heads, head_dim, bits, s_sink, s_keep, s_flush,
                 kappa_k, kappa_v, max_seq_len, win_slots=None, page_order="linear",
                 pool_factor=1.0, seed=0, device="cuda", codec="pclip", quest_alpha=None,
                 n_pages=None):
        torch = _torch()
        self.batch, self.n_kv_heads, self.head_dim, self.bits = batch, n_kv_heads, head_dim, bits
        self.s_sink, self.s_keep, self.s_flush = s_sink, s_keep, s_flush
        self.kappa_k, self.kappa_v = float(kappa_k), float(kappa_v)
        codes = {"pclip": _lib.CODEC_PCLIP, "quest": _lib.CODEC_QUEST}
        if codec not in codes:
            raise ValueError(codec)
        self.codec = codec
        if quest_alpha is None:
            quest_alpha = wushkv_quest_alpha(bits) if codec == "quest" else 0.0
        self.quest_alpha = float(ctypes.c_float(quest_alpha).value)  # as the descriptor holds it
        self.max_seq_len = max_seq_len
        if win_slots is None:
            need = s_sink + max(1, s_keep + s_flush - 1)
            win_slots = PAGE_TOKENS * math.ceil(need / PAGE_TOKENS)
        self.win_slots = win_slots
        self.max_pages = max(1, math.ceil(max(0, max_seq_len - s_sink) / PAGE_TOKENS))
        need_pages = batch * self.max_pages
        self.n_pages = max(need_pages, int(math.ceil(need_pages * pool_factor)))
        if n_pages is not None:
            if page_order != "none":
                raise ValueError("n_pages goes with page_order=\"none\"")
            self.n_pages = int(n_pages)
        self.page_bytes = wushkv_page_bytes(head_dim, bits)
        if self.page_bytes == 0:
            raise WushKVError(_lib.EUNSUPPORTED, "WushKVCache")
        dev = torch.device(device)
        self.device = dev
        self.pages = torch.zeros(self.n_pages * n_kv_heads * self.page_bytes, dtype=torch.uint8,
                                 device=dev)
        if page_order == "linear":
            table = torch.arange(need_pages, dtype=torch.int32)
        elif page_order == "random":
            g = torch.Generator().manual_seed(seed)
            table = torch.randperm(self.n_pages, generator=g)[:need_pages].to(torch.int32)
        elif page_order == "none":
            table = torch.full((need_pages,), -1, dtype=torch.int32)
        else:
            raise ValueError(page_order)
        self.page_table = table.reshape(batch, self.max_pages).contiguous().to(dev)
        self.win_k = torch.zeros(batch, n_kv_heads, win_slots, head_dim, dtype=torch.bfloat16,
                                 device=dev)
        self.win_v = torch.zeros(batch, n_kv_heads, head_dim, win_slots, dtype=torch.bfloat16,
                                 device=dev)
        self.seq_len = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.quant_end = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.commit = torch.zeros(batch, dtype=torch.int32, device=dev)
        self._desc = self._make_desc()

    def _make_desc(self) -> CacheDesc:
        return CacheDesc(
            self.batch, self.n_kv_heads, self.head_dim, self.bits, self.s_sink, self.s_keep,
            self.s_flush, self.win_slots, self.max_pages, self.n_pages, self.kappa_k,
            self.kappa_v, {"pclip": _lib.CODEC_PCLIP, "quest": _lib.CODEC_QUEST}[self.codec],
            self.quest_alpha, self.pages.data_ptr(), self.page_table.data_ptr(),
            self.win_k.data_ptr(), self.win_v.data_ptr(), self.seq_len.data_ptr(),
            self.quant_end.data_ptr(), self.commit.data_ptr())

    @property
    def desc(self) -> CacheDesc:
        return self._desc

    def clone(self) -> "WushKVCache":
        """Deep copy (same layout, same page table, fresh device memory)."""
        new = object.__new__(WushKVCache)
        new.__dict__.update({k: v for k, v in self.__dict__.items() if k != "_desc"})
        for name in ("pages", "page_table", "win_k", "win_v", "seq_len", "quant_end", "commit"):
            setattr(new, name, getattr(self, name).clone())
        new._desc = new._make_desc()
        return new


class WushKVBounds(_Described):
    """The boxes of a cache's complete pages (wushkv_page_bounds): ``codes``
    int8 [n_pages][n_kv][2][d], centres then radii, and ``scales`` fp32
    [n_kv][n_pages], zero-initialised on the cache's device."""

    def __init__(self, cache: WushKVCache):
        torch = _torch()
        self.codes = torch.zeros(cache.n_pages, cache.n_kv_heads, 2, cache.head_dim, dtype=torch.int8,
                                 device=cache.device)
        self.scales = torch.zeros(cache.n_kv_heads, cache.n_pages, dtype=torch.float32, device=cache.device)
        self._of = (cache.n_pages, cache.n_kv_heads, cache.head_dim, self.codes.get_device())
        self._desc = BoundsDesc(self.codes.data_ptr(), self.scales.data_ptr())

    @property
    def desc(self) -> BoundsDesc:
        return self._desc


class WushKVPool(_Described):
    """The bookkeeping of a cache's pages (wushkv_assign_pages): ``refs`` int32
    [n_pages], ``held`` int32 [batch] and ``low`` int32 [1].  Starts from the
    cache's page table: every entry of it is one reference, and a sequence holds
    what lies up to its last page and its last quantised position (evicted pages
    leave holes, which are given no page again)."""

    def __init__(self, cache: WushKVCache):
        torch = _torch()
        there = (cache.page_table >= 0) & (cache.page_table < cache.n_pages)
        number = torch.arange(1, cache.max_pages + 1, dtype=torch.int32, device=cache.device)
        positions = torch.minimum(cache.quant_end, cache.seq_len) - cache.s_sink
        stored = torch.div(positions + PAGE_TOKENS - 1, PAGE_TOKENS, rounding_mode="floor").clamp(0, cache.max_pages)
        self.held = torch.maximum((there * number).amax(1), stored.to(torch.int32))
        pages = cache.page_table[there].long()
        self.refs = torch.bincount(pages, minlength=cache.n_pages).to(torch.int32)
        self.low = torch.zeros(1, dtype=torch.int32, device=cache.device)
        self._of = (cache.n_pages, cache.batch, self.refs.get_device())
        self._desc = PoolDesc(self.refs.data_ptr(), self.held.data_ptr(), self.low.data_ptr())

    @property
    def desc(self) -> PoolDesc:
        return self._desc


def _check_2byte(t, name):
    if t is None:
        return
    if t.element_size() != 2 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 2-byte (bf16) tensor" % name)


def wushkv_append(cache: WushKVCache, k_new, v_new, n_new, t_k, k_tilde_out=None,
                  max_new=None, stream=None) -> None:
    """Alg. 2 steps 3-4 and 7-11 on the GPU.  k_new / v_new: bf16
    [batch][max_new][n_kv][d]; n_new: int32 [batch] on the device; t_k: bf16
    [n_kv][d][d]."""
    for t, nm in ((k_new, "k_new"), (v_new, "v_new"), (t_k, "t_k"), (k_tilde_out, "k_tilde_out")):
        _check_2byte(t, nm)
    if max_new is None:
        max_new = k_new.shape[1]
    st = _lib.lib().wushkv_append(ctypes.byref(cache.desc), _ptr(k_new), _ptr(v_new),
                                  _ptr(n_new), int(max_new), _ptr(t_k), _ptr(k_tilde_out),
                                  _stream_handle(stream))
    check(st, "wushkv_append")


def wushkv_append_norm_rope(cache: WushKVCache, k_raw, v_new, n_new, t_k, rope_table,
                            norm_gain=None, norm_eps=0.0, k_tilde_out=None, max_new=None,
                            stream=None) -> None:
    """wushkv_append with the headwise RMS normalisation and the rotary
    embedding of the new keys fused in front (Alg. 2 step 1).  k_raw: bf16
    [batch][max_new][n_kv][d] projected keys; rope_table: fp32 [positions][d]
    (cos | sin); norm_gain: fp32 [d] or None."""
    for t, nm in ((k_raw, "k_raw"), (v_new, "v_new"), (t_k, "t_k"), (k_tilde_out, "k_tilde_out")):
        _check_2byte(t, nm)
    if rope_table.element_size() != 4 or not rope_table.is_contiguous():
        raise ValueError("rope_table must be a contiguous fp32 tensor")
    if max_new is None:
        max_new = k_raw.shape[1]
    st = _lib.lib().wushkv_append_norm_rope(
        ctypes.byref(cache.desc), _ptr(k_raw), _ptr(v_new), _ptr(n_new), int(max_new), _ptr(t_k),
        _ptr(norm_gain), float(norm_eps), _ptr(rope_table), int(rope_table.shape[0]),
        _ptr(k_tilde_out), _stream_handle(stream))
    check(st, "wushkv_append_norm_rope")


def _decode_need(cache, n_q, max_seq_len) -> int:
    """The workspace size, or the error for sizes that have no plan (only
    asked for where no workspace is given, or after a call was refused: the
    library checks a given workspace itself)."""
    need = wushkv_decode_workspace_bytes(cache, n_q, max_seq_len)
    if need == 0:
        raise WushKVError(_lib.EINVAL, "wushkv_decode_workspace_bytes")
    return need


def _chunk_need(cache, n_q, max_tok, max_seq_len) -> int:
    need = wushkv_chunk_workspace_bytes(cache, n_q, max_tok, max_seq_len)
    if need == 0:
        raise WushKVError(_lib.EINVAL, "wushkv_chunk_workspace_bytes")
    return need


def wushkv_decode_workspace_bytes(cache: WushKVCache, n_q_heads: int, max_seq_len: int) -> int:
    return _lib.lib().wushkv_decode_workspace_bytes(ctypes.byref(cache.desc), n_q_heads,
                                                    max_seq_len)


def wushkv_decode_attention(cache: WushKVCache, q, t_k_inv, sm_scale=None, max_seq_len=None,
                            out=None, workspace=None, stream=None):
    """One decode query per query head.  q: bf16 [batch][n_q][d];
    t_k_inv: fp32 [n_kv][d][d].  Returns fp32 [batch][n_q][d]."""
    torch = _torch()
    _check_2byte(q, "q")
    n_q = q.shape[1]
    if max_seq_len is None:
        max_seq_len = cache.max_seq_len
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(cache.head_dim)
    if out is None:
        out = _on_stream(lambda: torch.empty(cache.batch, n_q, cache.head_dim, dtype=torch.float32, device=q.device),
                         stream)
    if workspace is None:
        need = _decode_need(cache, n_q, max_seq_len)
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=q.device), stream)
    st = _lib.lib().wushkv_decode_attention(
        ctypes.byref(cache.desc), _ptr(q), n_q, operator.index(max_seq_len), _ptr(t_k_inv),
        float(sm_scale), _ptr(out), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream_handle(stream))
    if st != _lib.OK:
        _decode_need(cache, n_q, max_seq_len)
        check(st, "wushkv_decode_attention")
    return out


def wushkv_decode_attention_noalloc(cache: WushKVCache, q, t_k_inv, out, sm_scale=None,
                                    max_seq_len=None, stream=None):
    """wushkv_decode_attention with the library's static workspace: nothing
    is allocated (``out`` is the caller's fp32 [batch][n_q][d]).  Calls that
    overlap on one GPU race on that workspace."""
    _check_2byte(q, "q")
    n_q = q.shape[1]
    if max_seq_len is None:
        max_seq_len = cache.max_seq_len
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(cache.head_dim)
    st = _lib.lib().wushkv_decode_attention_noalloc(
        ctypes.byref(cache.desc), _ptr(q), n_q, int(max_seq_len), _ptr(t_k_inv),
        float(sm_scale), _ptr(out), _stream_handle(stream))
    check(st, "wushkv_decode_attention_noalloc")
    return out


def wushkv_decode_step(cache: WushKVCache, k_new, v_new, n_new, t_k, q, t_k_inv, sm_scale=None,
                       max_seq_len=None, out=None, workspace=None, stream=None):
    """One decode step in Alg. 2's order: each sequence's new token (n_new[b]
    of 0 or 1) is appended, attention runs over the cache with it (the
    positions due for quantisation still at bf16), then the flush.
    k_new, v_new: bf16 [batch][n_kv][d]; n_new: int32 [batch] on the device;
    t_k: bf16 [n_kv][d][d]; q: bf16 [batch][n_q][d]; t_k_inv: fp32
    [n_kv][d][d].  Returns fp32 [batch][n_q][d]."""
    torch = _torch()
    _check_2byte(q, "q")
    _check_2byte(k_new, "k_new")
    _check_2byte(v_new, "v_new")
    _check_2byte(t_k, "t_k")
    n_q = q.shape[1]
    if max_seq_len is None:
        max_seq_len = cache.max_seq_len
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(cache.head_dim)
    if out is None:
        out = _on_stream(lambda: torch.empty(cache.batch, n_q, cache.head_dim, dtype=torch.float32, device=q.device),
                         stream)
    if workspace is None:
        need = _decode_need(cache, n_q, max_seq_len)
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=q.device), stream)
    st = _lib.lib().wushkv_decode_step(
        ctypes.byref(cache.desc), _ptr(k_new), _ptr(v_new), _ptr(n_new), _ptr(t_k), _ptr(q), n_q,
        operator.index(max_seq_len), _ptr(t_k_inv), float(sm_scale), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if st != _lib.OK:
        _decode_need(cache, n_q, max_seq_len)
        check(st, "wushkv_decode_step")
    return out


def wushkv_chunk_workspace_bytes(cache: WushKVCache, n_q_heads: int, max_tok: int,
                                 max_seq_len: int) -> int:
    return _lib.lib().wushkv_chunk_workspace_bytes(ctypes.byref(cache.desc), n_q_heads, max_tok,
                                                   max_seq_len)


def wushkv_chunk_attention(cache: WushKVCache, q, t_k_inv, n_tok=None, sm_scale=None,
                           max_seq_len=None, out=None, workspace=None, stream=None):
    """Attention of each sequence's chunk of new tokens, causal inside the
    chunk.  q: bf16 [batch][max_tok][n_q][d]; n_tok: int32 [batch] on the
    device or None (max_tok for all).  Returns fp32 [batch][max_tok][n_q][d]."""
    torch = _torch()
    _check_2byte(q, "q")
    max_tok, n_q = q.shape[1], q.shape[2]
    if max_seq_len is None:
        max_seq_len = cache.max_seq_len
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(cache.head_dim)
    if out is None:
        out = _on_stream(lambda: torch.empty(cache.batch, max_tok, n_q, cache.head_dim, dtype=torch.float32,
                                             device=q.device), stream)
    if workspace is None:
        need = _chunk_need(cache, n_q, max_tok, max_seq_len)
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=q.device), stream)
    st = _lib.lib().wushkv_chunk_attention(
        ctypes.byref(cache.desc), _ptr(q), _ptr(n_tok), int(max_tok), n_q, operator.index(max_seq_len),
        _ptr(t_k_inv), float(sm_scale), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if st != _lib.OK:
        _chunk_need(cache, n_q, max_tok, max_seq_len)
        check(st, "wushkv_chunk_attention")
    return out


def wushkv_dequant(cache: WushKVCache, b: int, start: int, count: int, k_out=None, v_out=None,
                   stream=None):
    """fp32 [n_kv][count][d] reconstructions of stored positions
    [start, start + count) of sequence b.  Returns (k_out, v_out)."""
    torch = _torch()
    shape = (cache.n_kv_heads, count, cache.head_dim)
    if k_out is None:
        k_out = _on_stream(lambda: torch.empty(shape, dtype=torch.float32, device=cache.device), stream)
    if v_out is None:
        v_out = _on_stream(lambda: torch.empty(shape, dtype=torch.float32, device=cache.device), stream)
    st = _lib.lib().wushkv_dequant(ctypes.byref(cache.desc), int(b), int(start), int(count),
                                   _ptr(k_out), _ptr(v_out), _stream_handle(stream))
    check(st, "wushkv_dequant")
    return k_out, v_out


def _check(dev, t, name, dtype, shape):
    """A contiguous tensor of this type and shape on device dev."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, list(shape)))
    if t.get_device() != dev:
        raise ValueError("%s is not on the cache's device" % name)
    return t.data_ptr()


def _check_space(dev, t):
    if not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("workspace must be contiguous and on the cache's device")
    return t.data_ptr(), t.numel() * t.element_size()


def _bounds_of(cache, dev, bounds):
    """Boxes of this cache's sizes, on its device."""
    if bounds._of != (cache.n_pages, cache.n_kv_heads, cache.head_dim, dev):
        raise ValueError("bounds are not this cache's")
    return ctypes.byref(bounds._desc)


def _pool_of(cache, dev, pool):
    """A pool of this cache's sizes, on its device."""
    if pool._of != (cache.n_pages, cache.batch, dev):
        raise ValueError("pool is not this cache's")
    return ctypes.byref(pool._desc)


def _launch_stream(dev, stream):
    """The stream handle of a call on device dev, which has to be the current
    one."""
    torch = _torch()
    current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)()
    if dev != current:
        raise ValueError("the cache's device is not the current one")
    if stream is not None:
        if stream.device_index != current:
            raise ValueError("the stream is not on the cache's device")
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(current) if raw is not None else torch.cuda.current_stream().cuda_stream


def _on_stream(make, stream):
    """A buffer made here for a call: on the call's stream, so that it is no block
    that another stream's launches still use, and kept until the current one, which
    may read it, has done with it."""
    if stream is None:
        return make()
    torch = _torch()
    now = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        t = make()
    if now != stream:
        t.record_stream(now)
    return t


def wushkv_page_bounds(cache: WushKVCache, bounds: WushKVBounds, since=None, max_new=None, stream=None) -> None:
    """The boxes of the pages completed since quant_end was ``since`` (int32
    [batch] on the device; None: of all complete pages), at most ``max_new``
    (by default max_pages) a sequence."""
    dev = cache.pages.get_device()
    box = _bounds_of(cache, dev, bounds)
    at = None if since is None else _check(dev, since, "since", _torch().int32, (cache.batch,))
    st = _lib.lib().wushkv_page_bounds(
        ctypes.byref(cache._desc), box, at, cache.max_pages if max_new is None else operator.index(max_new),
        _launch_stream(dev, stream))
    check(st, "wushkv_page_bounds")


def wushkv_select_workspace_bytes(cache: WushKVCache, n_q_heads: int, max_seq_len: int, top_k: int) -> int:
    return _lib.lib().wushkv_select_workspace_bytes(ctypes.byref(cache.desc), n_q_heads, max_seq_len, top_k)


def wushkv_select_pages(cache: WushKVCache, bounds: WushKVBounds, q, t_k_inv, top_k, max_seq_len=None, sel=None,
                        n_sel=None, scores=None, workspace=None, stream=None):
    """For each (sequence, kv head) the ``top_k`` complete pages with the
    largest bound on a logit of the query, and the page being filled.  q: bf16
    [batch][n_q][d]; t_k_inv: fp32 [n_kv][d][d].  Returns (sel int32
    [batch][n_kv][top_k + 1], ascending, -1 behind; n_sel int32
    [batch][n_kv]); ``scores``, if given, fp32 [batch][n_kv][max_pages],
    receives every complete page's score."""
    torch = _torch()
    dev = cache.pages.get_device()
    b, hk, d, top_k = cache.batch, cache.n_kv_heads, cache.head_dim, operator.index(top_k)
    n_q = q.shape[1] if q.dim() == 3 else 0
    box = _bounds_of(cache, dev, bounds)
    q_at = _check(dev, q, "q", torch.bfloat16, (b, n_q, d))
    t_at = _check(dev, t_k_inv, "t_k_inv", torch.float32, (hk, d, d))
    scores_at = None if scores is None else _check(dev, scores, "scores", torch.float32, (b, hk, cache.max_pages))
    max_seq_len = cache.max_seq_len if max_seq_len is None else operator.index(max_seq_len)
    if workspace is not None:
        space = _check_space(dev, workspace)
    handle = _launch_stream(dev, stream)
    if workspace is None:
        need = wushkv_select_workspace_bytes(cache, n_q, max_seq_len, top_k)
        if need == 0:
            raise WushKVError(_lib.EINVAL, "wushkv_select_workspace_bytes")
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=q.device), stream)
        space = workspace.data_ptr(), need
    shape = (b, hk, top_k + 1)
    if sel is None:
        sel = _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=q.device), stream)
    if n_sel is None:
        n_sel = _on_stream(lambda: torch.empty(b, hk, dtype=torch.int32, device=q.device), stream)
    st = _lib.lib().wushkv_select_pages(
        ctypes.byref(cache._desc), box, q_at, n_q, max_seq_len, t_at, top_k, _check(dev, sel, "sel", torch.int32, shape),
        _check(dev, n_sel, "n_sel", torch.int32, (b, hk)), scores_at, space[0], space[1], handle)
    check(st, "wushkv_select_pages")
    return sel, n_sel


def wushkv_sparse_workspace_bytes(cache: WushKVCache, n_q_heads: int, max_sel: int) -> int:
    return _lib.lib().wushkv_sparse_workspace_bytes(ctypes.byref(cache.desc), n_q_heads, max_sel)


def wushkv_sparse_attention(cache: WushKVCache, q, t_k_inv, sel, n_sel, sm_scale=None, out=None, workspace=None,
                            stream=None):
    """wushkv_decode_attention over the sink, the recent window and the listed
    pages: sel int32 [batch][n_kv][max_sel] logical pages, of which the first
    n_sel (int32 [batch][n_kv]) count.  Returns fp32 [batch][n_q][d]."""
    torch = _torch()
    dev = cache.pages.get_device()
    b, hk, d = cache.batch, cache.n_kv_heads, cache.head_dim
    n_q = q.shape[1] if q.dim() == 3 else 0
    max_sel = sel.shape[2] if sel.dim() == 3 else 0
    q_at = _check(dev, q, "q", torch.bfloat16, (b, n_q, d))
    t_at = _check(dev, t_k_inv, "t_k_inv", torch.float32, (hk, d, d))
    sel_at = _check(dev, sel, "sel", torch.int32, (b, hk, max_sel))
    n_at = _check(dev, n_sel, "n_sel", torch.int32, (b, hk))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    if workspace is not None:
        space = _check_space(dev, workspace)
    handle = _launch_stream(dev, stream)
    if out is None:
        out = _on_stream(lambda: torch.empty(b, n_q, d, dtype=torch.float32, device=q.device), stream)
    if workspace is None:
        # (sizes without a plan: the call says what is wrong)
        need = max(16, wushkv_sparse_workspace_bytes(cache, n_q, max_sel))
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=q.device), stream)
        space = workspace.data_ptr(), need
    st = _lib.lib().wushkv_sparse_attention(
        ctypes.byref(cache._desc), q_at, n_q, sel_at, n_at, max_sel, t_at, float(sm_scale),
        _check(dev, out, "out", torch.float32, (b, n_q, d)), space[0], space[1], handle)
    check(st, "wushkv_sparse_attention")
    return out


def wushkv_assign_pages(cache: WushKVCache, pool: WushKVPool, source=None, reach=None, status=None, stream=None):
    """Frees, forks and extends sequences: source[b] = b keeps sequence b, -1
    frees it, s makes it a copy of the kept sequence s (None keeps all);
    reach[b]: positions it is to hold pages for (None: no new ones).  Both
    int32 [batch] on the device.  Returns status int32 [batch]: pages missing,
    or -1 minus that where source[b] was refused.  A copy whose page being
    filled is missing (64 held < quantised positions) is freed, or copied from a
    whole sequence again, before it is given pages, appended to or forked."""
    torch = _torch()
    dev, shape = cache.pages.get_device(), (cache.batch,)
    books = _pool_of(cache, dev, pool)
    source_at = None if source is None else _check(dev, source, "source", torch.int32, shape)
    reach_at = None if reach is None else _check(dev, reach, "reach", torch.int32, shape)
    handle = _launch_stream(dev, stream)
    if status is None:
        status = _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=cache.device), stream)
    st = _lib.lib().wushkv_assign_pages(ctypes.byref(cache._desc), books, source_at, reach_at,
                                        _check(dev, status, "status", torch.int32, shape), handle)
    check(st, "wushkv_assign_pages")
    return status


def wushkv_compact_workspace_bytes(cache: WushKVCache) -> int:
    return _lib.lib().wushkv_compact_workspace_bytes(ctypes.byref(cache.desc))


def wushkv_compact_pages(cache: WushKVCache, pool: WushKVPool, bounds=None, table_out=None, refs_out=None,
                         live_out=None, workspace=None, stream=None):
    """Moves the n pages in use to the physical pages 0 .. n - 1 (with their
    boxes, if bounds is given).  The page table and references change in place
    or, where table_out and refs_out are given, into those, which the caller
    then swaps in (cache.page_table, pool.refs = table_out, refs_out) or copies
    over.  Returns (page table, references, n as int32 [1]), on the device."""
    torch = _torch()
    dev = cache.pages.get_device()
    books = _pool_of(cache, dev, pool)
    box = None if bounds is None else _bounds_of(cache, dev, bounds)
    if workspace is not None:
        space = _check_space(dev, workspace)
    handle = _launch_stream(dev, stream)
    if table_out is None:
        table_out = cache.page_table
    if refs_out is None:
        refs_out = pool.refs
    if live_out is None:
        live_out = _on_stream(lambda: torch.empty(1, dtype=torch.int32, device=cache.device), stream)
    if workspace is None:
        need = max(16, wushkv_compact_workspace_bytes(cache))
        workspace = _on_stream(lambda: torch.empty(need, dtype=torch.uint8, device=cache.device), stream)
        space = workspace.data_ptr(), need
    st = _lib.lib().wushkv_compact_pages(
        ctypes.byref(cache._desc), books, box,
        _check(dev, table_out, "table_out", torch.int32, (cache.batch, cache.max_pages)),
        _check(dev, refs_out, "refs_out", torch.int32, (cache.n_pages,)),
        _check(dev, live_out, "live_out", torch.int32, (1,)), space[0], space[1], handle)
    check(st, "wushkv_compact_pages")
    return table_out, refs_out, live_out


def wushkv_shared_prefixes(cache: WushKVCache, leader=None, shared=None, min_pages=1, stream=None):
    """The pages that sequences have in common at their start, from the page
    table: (leader, shared), int32 [batch] on the device, as
    wushkv_prefix_attention takes them; prefixes of fewer than ``min_pages``
    pages are left out.  They hold until a sequence that shares pages is freed
    or forked, or loses one of them."""
    torch = _torch()
    dev, shape = cache.pages.get_device(), (cache.batch,)
    min_pages = operator.index(min_pages)
    handle = _launch_stream(dev, stream)
    if leader is None:
        leader = _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=cache.device), stream)
    if shared is None:
        shared = _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=cache.device), stream)
    st = _lib.lib().wushkv_shared_prefixes(ctypes.byref(cache._desc), min_pages,
                                           _check(dev, leader, "leader", torch.int32, shape),
                                           _check(dev, shared, "shared", torch.int32, shape), handle)
    check(st, "wushkv_shared_prefixes")
    return leader, shared


def _rows_call(q, out, workspace, need, stream):
    """(out, its address, the workspace, its address and bytes): those given, or new
    ones; ``need`` gives the workspace's bytes, 0 where the call has no plan.  The
    caller keeps both until the library has been called: the block of a tensor that is
    gone may go to another thread's call before this one's launches."""
    torch = _torch()
    if out is None:
        out = _on_stream(lambda: torch.empty(q.shape, dtype=torch.float32, device=q.device), stream)
    out_at = _check(q.get_device(), out, "out", torch.float32, q.shape)
    if workspace is not None:
        return out, out_at, workspace, _check_space(q.get_device(), workspace)
    # (sizes without a plan: the call says what is wrong)
    n = max(16, need())
    workspace = _on_stream(lambda: torch.empty(n, dtype=torch.uint8, device=q.device), stream)
    return out, out_at, workspace, (workspace.data_ptr(), n)


def wushkv_prefix_workspace_bytes(cache: WushKVCache, n_q_heads: int) -> int:
    return _lib.lib().wushkv_prefix_workspace_bytes(ctypes.byref(cache.desc), n_q_heads)


def wushkv_prefix_attention(cache: WushKVCache, q, t_k_inv, leader, shared, sm_scale=None, out=None, workspace=None,
                            stream=None):
    """wushkv_decode_attention for sequences that share pages at their start,
    which are attended to together, 16 query rows at a time: leader, shared int32
    [batch] (wushkv_shared_prefixes).  The faster of the two where most of what the
    batch attends to is shared.  q: bf16 [batch][n_q][d]; t_k_inv: fp32
    [n_kv][d][d].  Returns fp32 [batch][n_q][d]."""
    torch = _torch()
    dev = cache.pages.get_device()
    b, hk, d = cache.batch, cache.n_kv_heads, cache.head_dim
    n_q = q.shape[1] if q.dim() == 3 else 0
    q_at = _check(dev, q, "q", torch.bfloat16, (b, n_q, d))
    t_at = _check(dev, t_k_inv, "t_k_inv", torch.float32, (hk, d, d))
    leader_at = _check(dev, leader, "leader", torch.int32, (b,))
    shared_at = _check(dev, shared, "shared", torch.int32, (b,))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    handle = _launch_stream(dev, stream)
    out, out_at, workspace, space = _rows_call(q, out, workspace, lambda: wushkv_prefix_workspace_bytes(cache, n_q), stream)
    st = _lib.lib().wushkv_prefix_attention(ctypes.byref(cache._desc), q_at, n_q, leader_at, shared_at, t_at,
                                            float(sm_scale), out_at, space[0], space[1], handle)
    check(st, "wushkv_prefix_attention")
    return out


def wushkv_cross_workspace_bytes(cache: WushKVCache, n_seqs: int, max_tok: int, n_q_heads: int) -> int:
    return _lib.lib().wushkv_cross_workspace_bytes(ctypes.byref(cache.desc), n_seqs, max_tok, n_q_heads)


def wushkv_cross_attention(cache: WushKVCache, q, t_k_inv, n_tok=None, source=None, sm_scale=None, out=None,
                           workspace=None, stream=None):
    """Attention of query sequences over whole stored ones, without a mask (a
    decoder's queries over an encoder's states).  q: bf16
    [n_seqs][max_tok][n_q][d]; n_tok: int32 [n_seqs] on the device or None
    (max_tok for all); source: int32 [n_seqs], the cache's sequence that each
    attends to (several may name the same), or None (its own number).  Returns
    fp32 [n_seqs][max_tok][n_q][d]."""
    torch = _torch()
    dev = cache.pages.get_device()
    hk, d = cache.n_kv_heads, cache.head_dim
    n_seqs, max_tok, n_q = q.shape[:3] if q.dim() == 4 else (0, 0, 0)
    q_at = _check(dev, q, "q", torch.bfloat16, (n_seqs, max_tok, n_q, d))
    t_at = _check(dev, t_k_inv, "t_k_inv", torch.float32, (hk, d, d))
    n_at = None if n_tok is None else _check(dev, n_tok, "n_tok", torch.int32, (n_seqs,))
    source_at = None if source is None else _check(dev, source, "source", torch.int32, (n_seqs,))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    handle = _launch_stream(dev, stream)
    out, out_at, workspace, space = _rows_call(
        q, out, workspace, lambda: wushkv_cross_workspace_bytes(cache, n_seqs, max_tok, n_q), stream)
    st = _lib.lib().wushkv_cross_attention(ctypes.byref(cache._desc), q_at, n_seqs, n_at, max_tok, source_at, n_q, t_at,
                                           float(sm_scale), out_at, space[0], space[1], handle)
    check(st, "wushkv_cross_attention")
    return out


def wushkv_weighted_workspace_bytes(cache: WushKVCache, n_q_heads: int, max_sel: int = -1) -> int:
    return _lib.lib().wushkv_weighted_workspace_bytes(ctypes.byref(cache.desc), n_q_heads, max_sel)


def wushkv_weighted_attention(cache: WushKVCache, q, t_k_inv, weights, sel=None, n_sel=None, sm_scale=None, out=None,
                              workspace=None, stream=None):
    """wushkv_sparse_attention over the listed pages (sel, n_sel), or over every
    page where both are None, that adds each page's attention weight to
    ``weights``, fp32 [batch][n_kv][max_pages].  Returns fp32 [batch][n_q][d]."""
    torch = _torch()
    dev = cache.pages.get_device()
    b, hk, d = cache.batch, cache.n_kv_heads, cache.head_dim
    n_q = q.shape[1] if q.dim() == 3 else 0
    q_at = _check(dev, q, "q", torch.bfloat16, (b, n_q, d))
    t_at = _check(dev, t_k_inv, "t_k_inv", torch.float32, (hk, d, d))
    w_at = _check(dev, weights, "weights", torch.float32, (b, hk, cache.max_pages))
    if (sel is None) != (n_sel is None):
        raise ValueError("sel and n_sel go together")
    max_sel, sel_at, n_at = -1, None, None
    if sel is not None:
        max_sel = sel.shape[2] if sel.dim() == 3 else 0
        sel_at = _check(dev, sel, "sel", torch.int32, (b, hk, max_sel))
        n_at = _check(dev, n_sel, "n_sel", torch.int32, (b, hk))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(d)
    handle = _launch_stream(dev, stream)
    out, out_at, workspace, space = _rows_call(
        q, out, workspace, lambda: wushkv_weighted_workspace_bytes(cache, n_q, max_sel), stream)
    st = _lib.lib().wushkv_weighted_attention(ctypes.byref(cache._desc), q_at, n_q, sel_at, n_at, max_sel, t_at,
                                              float(sm_scale), w_at, out_at, space[0], space[1], handle)
    check(st, "wushkv_weighted_attention")
    return out


def wushkv_evict_pages(cache: WushKVCache, pool: WushKVPool, weights, budget, recent=0, max_sel=None, sel=None,
                       n_sel=None, table_out=None, refs_out=None, evicted=None, stream=None):
    """The complete pages with the least weight (fp32 [batch][n_kv][max_pages])
    leave each sequence b that has more than budget[b] (int32 [batch]; negative:
    as it is), but for its newest ``recent``.  The page table and references
    change in place or, where table_out and refs_out are given, into those.
    Returns (sel int32 [batch][n_kv][max_sel], the pages left, ascending, -1
    behind; n_sel int32 [batch][n_kv]; evicted int32 [batch])."""
    torch = _torch()
    dev = cache.pages.get_device()
    books = _pool_of(cache, dev, pool)
    b, hk = cache.batch, cache.n_kv_heads
    w_at = _check(dev, weights, "weights", torch.float32, (b, hk, cache.max_pages))
    budget_at = _check(dev, budget, "budget", torch.int32, (b,))
    if sel is not None:
        if max_sel is not None and sel.shape[-1] != operator.index(max_sel):
            raise ValueError("sel has another width than max_sel")
        max_sel = sel.shape[2] if sel.dim() == 3 else 0
    max_sel = cache.max_pages if max_sel is None else operator.index(max_sel)
    handle = _launch_stream(dev, stream)
    new = lambda *shape: _on_stream(lambda: torch.empty(shape, dtype=torch.int32, device=cache.device), stream)  # noqa: E731
    if sel is None:
        sel = new(b, hk, max(max_sel, 0))
    if n_sel is None:
        n_sel = new(b, hk)
    if evicted is None:
        evicted = new(b)
    if table_out is None:
        table_out = cache.page_table
    if refs_out is None:
        refs_out = pool.refs
    sel_at = _check(dev, sel, "sel", torch.int32, (b, hk, max(max_sel, 0)))
    st = _lib.lib().wushkv_evict_pages(
        ctypes.byref(cache._desc), books, w_at, budget_at, operator.index(recent),
        _check(dev, table_out, "table_out", torch.int32, (b, cache.max_pages)),
        _check(dev, refs_out, "refs_out", torch.int32, (cache.n_pages,)),
        # (lists of no entries have no address, their counts have)
        sel_at if max_sel > 0 else None, _check(dev, n_sel, "n_sel", torch.int32, (b, hk)), max_sel,
        _check(dev, evicted, "evicted", torch.int32, (b,)), handle)
    check(st, "wushkv_evict_pages")
    return sel, n_sel, evicted


def wushkv_wush_transform(m, h, gamma: float = 1e-2, t_out=None, t_inv_out=None,
                          want_inverse: bool = True, sweeps_out=None, stream=None):
    """T = Wush(M, H, gamma) of Eq. (1) for each of the [count][d][d] fp32
    (device, symmetric) pairs in m and h.  Returns (T, T^{-1} or None,
    sweeps int32 [count]: Jacobi sweeps taken, -1 where a damped matrix was
    not positive definite)."""
    torch = _torch()
    if m.shape != h.shape or m.dim() != 3 or m.shape[1] != m.shape[2]:
        raise ValueError("m and h must both be [count][d][d]")
    count, d = int(m.shape[0]), int(m.shape[1])
    for t in (m, h):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("m and h must be contiguous fp32")
    if t_out is None:
        t_out = _on_stream(lambda: torch.empty_like(m), stream)
    if want_inverse and t_inv_out is None:
        t_inv_out = _on_stream(lambda: torch.empty_like(m), stream)
    if sweeps_out is None:
        sweeps_out = _on_stream(lambda: torch.empty(count, dtype=torch.int32, device=m.device), stream)
    st = _lib.lib().wushkv_wush_transform(_ptr(m), _ptr(h), count, d, float(gamma), _ptr(t_out),
                                          _ptr(t_inv_out) if want_inverse else None,
                                          _ptr(sweeps_out), _stream_handle(stream))
    check(st, "wushkv_wush_transform")
    return t_out, (t_inv_out if want_inverse else None), sweeps_out


def wushkv_read_probe(buf, mode: int, sink=None, stream=None):
    """Streaming read of the device tensor buf (byte size a multiple of
    65536), mode 0 vector loads or 1 direct-to-LDS loads.  Returns sink."""
    torch = _torch()
    nbytes = buf.numel() * buf.element_size()
    if sink is None:
        sink = _on_stream(lambda: torch.empty(max(1, nbytes // 65536), dtype=torch.int32, device=buf.device), stream)
    check(_lib.lib().wushkv_read_probe(_ptr(buf), nbytes, int(mode), _ptr(sink),
                                       _stream_handle(stream)), "wushkv_read_probe")
    return sink
