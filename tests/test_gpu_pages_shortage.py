"""A fork that did not get its own page: attention leaves its positions out, and
as a copy of the whole sequence again it is the same as that."""
import numpy as np
import pytest
import torch

import pages_ref
import paper_2609_38121_amd as wk
from gpu_harness import rel_err
from pages_ref import Host, transform
from sparse_exact import off, rows
from test_gpu_pages import bf16, dev_i32, same_state
from test_gpu_sparse import run
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,bits", [(64, 2), (128, 4)])
def test_a_fork_without_its_own_page(gpu, d, bits):
    rng = np.random.default_rng([d, bits, 9])
    h = Host(rng, [500, 0, 200], 2, d, bits, spare=0)
    c, pool = h.cache(gpu)
    q = synth.to_bf16_bits(rng.standard_normal((3, 4, d)))
    q[1] = q[0]
    t = transform(rng, 2, d)
    sel = np.broadcast_to(np.arange(h.max_pages, dtype=np.int32), (3, 2, h.max_pages)).copy()
    n = np.full((3, 2), h.max_pages, np.int32)

    def assign(source):
        status = wk.wushkv_assign_pages(c, pool, source=dev_i32(source, gpu)).cpu().numpy()
        assert np.array_equal(status, pages_ref.assign(h, source))
        same_state(c, pool, h)
        return status.tolist()

    def attend():
        got = run(gpu, h, q, t, sel, n, cache=c)
        most, rms = off(got, *rows(h, q, t, sel, n))
        assert most <= 1.0 and rms <= 1.0
        dense = wk.wushkv_decode_attention(c, bf16(q, gpu), torch.from_numpy(t).to(gpu)).cpu().numpy()
        assert rel_err(got, dense) <= 1e-3
        return got, dense

    assert assign([0, 0, 2]) == [0, 1, 0]
    assert 64 * h.held[1] < h.end(1) - 4  # how such a fork is told from others
    attend()
    assert assign([0, 0, -1]) == [0, 0, 0]
    for out in attend():
        assert np.array_equal(out[0], out[1])
