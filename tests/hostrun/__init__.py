"""csrc/pages.hip compiled for the host (common.h here), its entry points over
numpy arrays."""
import ctypes
import os
import shutil
import subprocess

import numpy as np

from paper_2609_38121_amd import _lib
from paper_2609_38121_amd.build import CSRC, HIPCC, INCLUDE

HERE = os.path.dirname(os.path.abspath(__file__))


def build(folder):
    """The library, built in this (scratch) folder."""
    for path in (os.path.join(HERE, "common.h"), os.path.join(HERE, "merge.h"), os.path.join(CSRC, "pages.hip")):
        shutil.copy(path, folder)
    so = os.path.join(folder, "libpages_host.so")
    compiler = os.path.join(os.path.dirname(os.path.realpath(shutil.which(HIPCC))), "amdclang++")
    subprocess.run([compiler, "-O2", "-std=c++17", "-fPIC", "-shared", "-x", "c++", "-I", INCLUDE,
                    os.path.join(folder, "pages.hip"), "-o", so], check=True)
    L = ctypes.CDLL(so)
    L.wushkv_compact_workspace_bytes.restype = ctypes.c_size_t
    return L


def array(a, dtype=np.int32):
    """A copy at an address that the entry points take."""
    a = np.asarray(a, dtype)
    room = np.empty(a.nbytes + 16, np.uint8)
    out = room[-room.ctypes.data % 16:][:a.nbytes].view(dtype).reshape(a.shape)
    out[...] = a
    return out


class State:
    """A cache and its pool, or what the two calls use of them, in host arrays:
    copies of those of ``of`` (a pages_ref.Host, or anything with its names)."""

    def __init__(self, of):
        self.b, self.hk, self.d, self.bits, self.s_sink = of.b, of.hk, of.d, of.bits, of.s_sink
        self.max_pages, self.n_pages = of.max_pages, of.n_pages
        for name in ("table", "refs", "held", "seq_len", "quant_end"):
            setattr(self, name, array(getattr(of, name)))
        self.pages = array(of.pages, np.uint8)
        self.win_k, self.win_v = array(of.win_k, np.uint16), array(of.win_v, np.uint16)
        self.low, self.commit = array([0]), array(np.zeros(of.b))
        self.win_slots = of.win_k.shape[2]

    def cache(self):
        at = lambda a: a.ctypes.data  # noqa: E731
        return _lib.CacheDesc(self.b, self.hk, self.d, self.bits, self.s_sink, 32, 8, self.win_slots, self.max_pages,
                              self.n_pages, 0.96, 0.92, _lib.CODEC_PCLIP, 0.0, at(self.pages), at(self.table),
                              at(self.win_k), at(self.win_v), at(self.seq_len), at(self.quant_end), at(self.commit))

    def pool(self):
        return _lib.PoolDesc(self.refs.ctypes.data, self.held.ctypes.data, self.low.ctypes.data)

    def assign(self, L, source=None, reach=None):
        status = array(np.full(self.b, 99))
        source, reach = (None if a is None else array(a) for a in (source, reach))
        st = L.wushkv_assign_pages(ctypes.byref(self.cache()), ctypes.byref(self.pool()),
                                   *(ctypes.c_void_p(None if a is None else a.ctypes.data) for a in (source, reach, status)),
                                   None)
        assert st == 0
        return status

    def compact(self, L, codes=None, scales=None, table_out=None, refs_out=None):
        c, p = self.cache(), self.pool()
        need = L.wushkv_compact_workspace_bytes(ctypes.byref(c))
        # (bytes of its own round the workspace, so that a wrong rank is an assertion; zeros name a page)
        guard = 16 * self.n_pages
        room, live = array(np.zeros(need + 2 * guard), np.uint8), array([-1])
        space = room[guard:guard + need]
        box = None if codes is None else ctypes.byref(_lib.BoundsDesc(codes.ctypes.data, scales.ctypes.data))
        out = (self.table if table_out is None else table_out, self.refs if refs_out is None else refs_out, live, space)
        st = L.wushkv_compact_pages(ctypes.byref(c), ctypes.byref(p), box,
                                    *(ctypes.c_void_p(a.ctypes.data) for a in out), ctypes.c_size_t(need), None)
        assert st == 0
        assert not room[:guard].any() and not room[guard + need:].any(), "a write outside the workspace"
        return int(live[0])
