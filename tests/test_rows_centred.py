"""The attentions of many query rows centre values on the middle of their codes, at
every width: sums that are exact that way, and in no other (tests/centred.py)."""
import numpy as np
import pytest
import torch

import centred
import pages_ref
import paper_2609_38121_amd as wk
from gpu_harness import say
from test_gpu_pages import dev_i32
from test_gpu_rows import f32, fork

LENS = [1500, 700, 1100, 333]


@pytest.mark.parametrize("d,bits", [(64, 2), (64, 3), (128, 4), (128, 3)])
def test_other_middles_are_outside(d, bits):
    h = centred.state(np.random.default_rng([d, bits]), LENS, 1, d, bits)
    want = np.stack([centred.row(h, b, 0) for b in range(4)])
    for middle in (0, 2, 4, 8):
        off = centred.off(np.stack([centred.fp32_row(h, b, 0, middle) for b in range(4)]), want)
        assert off <= 1.0 if middle == 1 << (bits - 1) else off > 8.0, (middle, off)


@pytest.mark.gpu
@pytest.mark.parametrize("d,bits,G,hk", [(64, 2, 2, 2), (64, 3, 4, 1), (128, 3, 8, 2), (128, 3, 1, 3), (128, 4, 4, 2), (64, 4, 1, 1),
                                         (128, 2, 8, 1)])
def test_sums_are_exact(gpu, d, bits, G, hk):
    say("exact sums, d %d, %d-bit, G %d, %d heads" % (d, bits, G, hk))
    rng = np.random.default_rng([d, bits, G, hk])
    h = centred.state(rng, LENS, hk, d, bits)
    fork(h, 2, 0, 9)
    c, _ = h.cache(gpu)
    t = f32(pages_ref.transform(rng, hk, d), gpu)
    want = np.repeat(np.stack([[centred.row(h, b, i) for i in range(hk)] for b in range(4)]), G, 1)
    q = torch.zeros(4, hk * G, d, dtype=torch.bfloat16, device=gpu)
    weights = torch.zeros(4, hk, h.max_pages, device=gpu)
    outs = {
        "weighted": wk.wushkv_weighted_attention(c, q, t, weights),
        "prefix": wk.wushkv_prefix_attention(c, q, t, dev_i32([0, 1, 0, 3], gpu), dev_i32([0, 0, 9, 0], gpu)),
        "cross": wk.wushkv_cross_attention(c, q[:, None].expand(4, 20, hk * G, d).contiguous(), t),
    }
    torch.cuda.synchronize()
    for name, out in outs.items():
        got = out.cpu().numpy().reshape(4, -1, hk * G, d)  # (cross: 20 tokens each)
        off = max(centred.off(got[:, i], want) for i in range(got.shape[1]))
        say("  %s: %.2f roundings" % (name, off))
        assert off <= 1.0
