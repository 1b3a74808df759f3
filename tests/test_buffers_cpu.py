"""The buffers that the binding makes for a call: alive until the library has been
called.  No GPU: the library's launches are replaced by functions that look at their
arguments, and the caches' arrays lie in host memory."""
import weakref

import pytest
import torch

wk = pytest.importorskip("paper_2609_38121_amd")
from paper_2609_38121_amd import _lib  # noqa: E402


class Torch:
    """torch, with a record of the tensors that are made through it."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return getattr(torch, name)

    def _record(self, t):
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
