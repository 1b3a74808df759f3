"""Calls on a stream given by hand, with every buffer left to the binding: the default
stream's results, and no block that the default stream's launches may still use."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
from pages_ref import Host
from test_gpu_pages import bf16, dev_i32
from test_gpu_rows import f32, queries

pytestmark = pytest.mark.gpu


def test_on_another_stream(gpu):
    rng = np.random.default_rng(12)
    h = Host(rng, [700, 333, 50], 2, 128, 2)
    c, _ = h.cache(gpu)
    q, t = queries(rng, 3, 8, 128), f32(pages_ref.transform(rng, 2, 128), gpu)
    q1, q4, n = bf16(q, gpu), bf16(queries(rng, 3, 5, 8, 128), gpu), dev_i32([5, 2, 0], gpu)
    square = torch.eye(128, device=gpu).repeat(2, 1, 1) + 0.01
    new, one, tk = bf16(queries(rng, 3, 2, 128), gpu), dev_i32([1, 1, 1], gpu), t.bfloat16()

    def run(stream, cache):
        return [wk.wushkv_decode_attention(cache, q1, t, stream=stream), wk.wushkv_chunk_attention(cache, q4, t, n, stream=stream),
                *wk.wushkv_dequant(cache, 0, 4, 500, stream=stream), *wk.wushkv_wush_transform(square, square, stream=stream),
                wk.wushkv_read_probe(cache.pages[:cache.pages.numel() // 65536 * 65536], 0, stream=stream),
                wk.wushkv_decode_step(cache, new, new, one, tk, q1, t, stream=stream)]

    want = run(None, c.clone())
    side, mine = torch.cuda.Stream(), c.clone()
    side.wait_stream(torch.cuda.current_stream())
    # blocks of every size that the calls make, back in the current stream's pool
    held = [torch.empty_like(x) for x in want for _ in range(2)]
    held += [torch.empty(n, dtype=torch.uint8, device=gpu) for n in (
        wk.wushkv_decode_workspace_bytes(c, 8, c.max_seq_len), wk.wushkv_chunk_workspace_bytes(c, 8, 5, c.max_seq_len))]
    before = {x.data_ptr() for x in held}
    del held
    got = run(side, mine)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not {x.data_ptr() for x in got} & before


def test_two_threads_on_one_stream(gpu):
    """Calls without a workspace from two threads: each call's is its own until its
    launches are enqueued."""
    import threading

    def make(seed):
        rng = np.random.default_rng(seed)
        h = Host(rng, [700, 333, 650, 50], 2, 128, 2)
        h.table[2, :6] = h.table[0, :6]
        c, _ = h.cache(gpu)
        q, x, t = bf16(queries(rng, 4, 8, 128), gpu), bf16(queries(rng, 4, 3, 8, 128), gpu), f32(pages_ref.transform(rng, 2, 128), gpu)
        leader, shared = wk.wushkv_shared_prefixes(c)
        w = torch.zeros(4, 2, h.max_pages, device=gpu)
        return lambda: (wk.wushkv_prefix_attention(c, q, t, leader, shared), wk.wushkv_cross_attention(c, x, t),
                        wk.wushkv_weighted_attention(c, q, t, w))

    calls = [make(s) for s in (1, 2)]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        for _ in range(100):
            got[i].append(calls[i]())

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(2):
        assert len(got[i]) == 100
        assert all(torch.equal(a, b) for run in got[i] for a, b in zip(run, want[i]))
