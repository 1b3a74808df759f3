"""The buffers that the binding makes for a call: alive until the library has been
called, and from the stream that it is given.  No GPU: the library's launches are
replaced by functions that look at their arguments, and the caches' arrays lie in host
memory."""
import contextlib
import types
import weakref

import pytest
import torch

wk = pytest.importorskip("paper_2609_38121_amd")
from paper_2609_38121_amd import _lib  # noqa: E402


class Made(torch.Tensor):
    """A tensor that remembers the streams whose use of it was recorded."""

    def record_stream(self, stream):
        self.used_on = getattr(self, "used_on", ()) + (stream,)


class Torch:
    """torch, with a record of the tensors that are made through it and of the stream
    that was the current one; "here" is where nothing else is said."""

    def __init__(self):
        self.made, self.now = [], "here"
        self.cuda = types.SimpleNamespace(current_stream=lambda device=None: self.now, stream=self._on)

    def __getattr__(self, name):
        return getattr(torch, name)

    @contextlib.contextmanager
    def _on(self, stream):
        was, self.now = self.now, stream
        yield
        self.now = was

    def _record(self, t):
        t = t.as_subclass(Made)
        t.made_on = self.now
        self.made.append((t.data_ptr(), weakref.ref(t)))
        return t

    def empty(self, *size, **kw):
        return self._record(torch.empty(*size, **kw))

    def empty_like(self, t, **kw):
        return self._record(torch.empty_like(t, **kw))


class Library:
    """The library's sizes; of its launches ``names`` go to ``call``."""

    def __init__(self, names, call):
        self.real, self.names, self.call = _lib.lib(), names, call

    def __getattr__(self, name):
        if name in self.names:
            return lambda *args: self.call(name, args)
        return getattr(self.real, name)


B, HK, G, D = 3, 2, 2, 64


def cache(**kw):
    return wk.WushKVCache(B, HK, D, 2, 4, 32, 8, 0.96, 0.92, max_seq_len=500, device="cpu", **kw)


def tensors():
    return (torch.zeros(B, HK * G, D, dtype=torch.bfloat16), torch.zeros(HK, D, D),
            lambda *shape: torch.zeros(shape, dtype=torch.int32))


def attentions():
    """name: the call, with every buffer left to the binding."""
    c, (q, t, ints) = cache(), tensors()
    weights = torch.zeros(B, HK, c.max_pages)
    return {
        "wushkv_prefix_attention": lambda: wk.wushkv_prefix_attention(c, q, t, ints(B), ints(B)),
        "wushkv_cross_attention": lambda: wk.wushkv_cross_attention(c, q[:, None].contiguous(), t),
        "wushkv_weighted_attention": lambda: wk.wushkv_weighted_attention(c, q, t, weights),
        "wushkv_sparse_attention": lambda: wk.wushkv_sparse_attention(c, q, t, ints(B, HK, 3), ints(B, HK)),
        "wushkv_decode_attention": lambda: wk.wushkv_decode_attention(c, q, t),
        "wushkv_chunk_attention": lambda: wk.wushkv_chunk_attention(c, q[:, None].contiguous(), t),
        "wushkv_select_pages": lambda: wk.wushkv_select_pages(c, wk.WushKVBounds(c), q, t, 3),
        "wushkv_compact_pages": lambda: wk.wushkv_compact_pages(c, wk.WushKVPool(c)),
    }


@pytest.mark.parametrize("name", sorted(attentions()))
def test_buffers_outlive_the_call(name, monkeypatch):
    """A block whose tensor is gone can be handed to another thread's call before this
    one's launches are enqueued."""
    seen = []
    fake = Torch()

    def call(_, args):
        made = dict(fake.made)
        here = [made[a] for a in args if isinstance(a, int) and a in made]
        seen.append([r() is not None for r in here])
        return 0

    call_it = attentions()[name]
    monkeypatch.setattr(wk, "_torch", lambda: fake)
    monkeypatch.setattr(wk, "_launch_stream", lambda dev, stream: 0)
    monkeypatch.setattr(wk, "_stream_handle", lambda stream: 0)
    monkeypatch.setattr(_lib, "lib", lambda lib=Library({name}, call): lib)
    call_it()
    # the output and the workspace at least, all of them alive
    assert len(seen) == 1 and len(seen[0]) >= 2 and all(seen[0])


class Stream:
    """A stream other than the current one."""
    cuda_stream, device, device_index = 77, torch.device("cpu"), -1


def streamed():
    """name: the call with a stream, with every buffer left to the binding."""
    c, (q, t, ints) = cache(), tensors()
    q4, new = q[:, None].contiguous(), torch.zeros(B, HK, D, dtype=torch.bfloat16)
    tk, weights, square = t.bfloat16(), torch.zeros(B, HK, c.max_pages), torch.zeros(2, D, D)
    return {
        "wushkv_prefix_attention": lambda s: wk.wushkv_prefix_attention(c, q, t, ints(B), ints(B), stream=s),
        "wushkv_cross_attention": lambda s: wk.wushkv_cross_attention(c, q4, t, stream=s),
        "wushkv_weighted_attention": lambda s: wk.wushkv_weighted_attention(c, q, t, weights, stream=s),
        "wushkv_sparse_attention": lambda s: wk.wushkv_sparse_attention(c, q, t, ints(B, HK, 3), ints(B, HK), stream=s),
        "wushkv_select_pages": lambda s: wk.wushkv_select_pages(c, wk.WushKVBounds(c), q, t, 3, stream=s),
        "wushkv_compact_pages": lambda s: wk.wushkv_compact_pages(c, wk.WushKVPool(c), stream=s),
        "wushkv_assign_pages": lambda s: wk.wushkv_assign_pages(c, wk.WushKVPool(c), stream=s),
        "wushkv_shared_prefixes": lambda s: wk.wushkv_shared_prefixes(c, stream=s),
        "wushkv_evict_pages": lambda s: wk.wushkv_evict_pages(c, wk.WushKVPool(c), weights, ints(B), stream=s),
        "wushkv_decode_attention": lambda s: wk.wushkv_decode_attention(c, q, t, stream=s),
        "wushkv_decode_step": lambda s: wk.wushkv_decode_step(c, new, new, ints(B), tk, q, t, stream=s),
        "wushkv_chunk_attention": lambda s: wk.wushkv_chunk_attention(c, q4, t, stream=s),
        "wushkv_dequant": lambda s: wk.wushkv_dequant(c, 0, 4, 64, stream=s),
        "wushkv_wush_transform": lambda s: wk.wushkv_wush_transform(square, square, stream=s),
        "wushkv_read_probe": lambda s: wk.wushkv_read_probe(torch.zeros(65536, dtype=torch.uint8), 0, stream=s),
    }


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("name", sorted(streamed()))
def test_buffers_come_from_the_calls_stream(name, given, monkeypatch):
    """A block of the current stream's pool may still be used by that stream's
    launches, which the call's stream does not wait for; what the call's stream gets
    back, the current one may still read."""
    seen, fake, side = [], Torch(), Stream()

    def call(_, args):
        made = dict(fake.made)
        seen.extend(made[a]() for a in args if isinstance(a, int) and a in made)
        return 0

    call_it = streamed()[name]
    monkeypatch.setattr(wk, "_torch", lambda: fake)
    monkeypatch.setattr(wk, "_launch_stream", lambda dev, stream: 0)
    monkeypatch.setattr(wk, "_stream_handle", lambda stream: 0)
    monkeypatch.setattr(_lib, "lib", lambda lib=Library({name}, call): lib)
    result = call_it(side if given else None)
    assert len(seen) >= 1 and None not in seen and result is not None
    for t in seen:
        assert t.made_on == (side if given else "here")
        assert getattr(t, "used_on", ()) == (("here",) if given else ())
