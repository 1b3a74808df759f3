"""Selections of rows beyond one workgroup's, up to more scores than its LDS
holds, against the plain form, value for value."""
import numpy as np
import pytest

import pages_ref
from gpu_harness import say
from pages_ref import Host
from test_gpu_pages import check_selection, random_boxes
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,G,pages,top_k,few", [(128, 8, 700, 90, False), (128, 1, 513, 512, False), (64, 8, 1300, 1, True),
                                                 (64, 2, 16384, 3000, False), (64, 2, 16385, 1, False),
                                                 (64, 1, 20000, 7001, True), (64, 1, 17000, 30000, False)])
def test_long_rows(gpu, d, G, pages, top_k, few):
    """few: scores with many equal among them."""
    say("d %d, G %d, %d pages, top %d" % (d, G, pages, top_k))
    rng = np.random.default_rng([d, G, pages])
    # all entries name a page of a small pool: the pages themselves are not read
    h = Host(rng, [200], 1, d, 2, spare=60 if not few else 3)
    h.seq_len = np.array([4 + 32 + 64 * pages + 9], np.int32)
    h.quant_end = (4 + (h.seq_len - 36) // 8 * 8).astype(np.int32)
    h.max_pages = pages + 1
    h.table = rng.integers(0, h.n_pages, (1, h.max_pages)).astype(np.int32)
    h.held = np.full(1, h.max_pages, np.int32)
    assert h.complete(0) == pages and h.every(0) == pages + 1
    codes, scales = random_boxes(rng, h)
    q = synth.to_bf16_bits(rng.standard_normal((1, G, d)))
    check_selection(gpu, h, codes, scales, q, pages_ref.transform(rng, 1, d), top_k)
