"""The tolerance of the listed attention has to be missed by a page left out and
by each loss of precision that the kernel takes a step against, planted in the
plain evaluation."""
import numpy as np
import pytest

import pages_ref
import sparse_exact


@pytest.mark.parametrize("name", sparse_exact.STATES)
@pytest.mark.parametrize("d,bits,G,slots", [(128, 4, 4, 64), (128, 2, 2, 64), (64, 4, 8, 192), (64, 2, 1, 64)])
def test_a_planted_mistake_is_outside(name, d, bits, G, slots):
    if name == "far zeros" and bits == 2:
        pytest.skip("2-bit codes reach 1.5 steps from the middle: hardly worse uncentred")
    s = sparse_exact.state(name, d, bits, G, 2, 3, slots)
    want, tol = sparse_exact.rows(*s)
    assert sparse_exact.off(want, want, tol) == (0.0, 0.0)
    wrong, _ = sparse_exact.rows(*s, plant=sparse_exact.STATES[name])
    most, rms = sparse_exact.off(wrong, want, tol)
    assert most > 1.0 and rms > 1.0, (most, rms)
    # far below an output's size, and the same evaluation as the other tests'
    size = np.linalg.norm(want, axis=-1)
    assert (3.0 * tol[0] + tol[1] <= 2e-5 * size).all()
    host, q, t, sel, n = s
    other, _ = pages_ref.attention(host, q, t, sel, n, 1.0 / np.sqrt(d))
    assert (np.linalg.norm(other - want, axis=-1) <= 1e-12 * size).all()
