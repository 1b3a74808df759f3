"""Which form a listed attention takes: a row in one workgroup only where its
list and its windows are short, or where the rows fill the device."""
import numpy as np
import pytest
import torch

import paper_2609_38121_amd as wk
from gpu_harness import say
from pages_ref import Host, transform
from sparse_exact import lists
from test_gpu_sparse_precision import close
from workloads import synth

pytestmark = pytest.mark.gpu


def kernels(gpu, h, q, t, sel, n):
    """The names of the attention launches of one call."""
    c, _ = h.cache(gpu)
    args = [torch.from_numpy(x).to(gpu) for x in (q.view(np.int16), t, sel, n)]
    wk.wushkv_timing_enable(8)
    try:
        wk.wushkv_sparse_attention(c, args[0].view(torch.bfloat16), *args[1:])
        torch.cuda.synchronize()
        return [name for name, _ in wk.wushkv_timing_launches() if name.startswith("sparse")]
    finally:
        wk.wushkv_timing_enable(0)


@pytest.mark.parametrize("d,slots,width,batch,one", [(64, 64, 8, 1, True), (64, 192, 8, 3, True), (64, 256, 8, 1, False),
                                                     (64, 2048, 3, 2, False), (64, 64, 9, 1, False), (128, 64, 1, 1, False),
                                                     (128, 64, 1, 150, True), (64, 512, 9, 150, True)])
def test_the_form_taken(gpu, d, slots, width, batch, one):
    say("d %d, %d slots, %d pages, %d sequences" % (d, slots, width, batch))
    rng = np.random.default_rng([d, slots, width, batch])
    keep = slots - 20
    h = Host(rng, [400 + keep, 33 + keep, keep // 2][:batch] + [20] * (batch - 3), 2, d, 2, s_keep=keep, win_slots=slots)
    q = synth.to_bf16_bits(rng.standard_normal((batch, 4, d)))
    t = transform(rng, 2, d)
    sel, n = lists(rng, h, width, least=1)
    assert kernels(gpu, h, q, t, sel, n) == ["sparse_row_kernel" if one else "sparse_main_kernel"]
    close(gpu, h, q, t, sel, n, pick=np.arange(min(batch, 3)), what="one workgroup a row" if one else "split")
