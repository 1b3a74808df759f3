"""The tolerance of the attentions of many query rows (tests/rows_close.py) has to be
missed by a page left out and by each loss of precision that the kernels take a step
against, planted in the plain evaluation in the state that shows it.

(The values' middle has a test of its own, tests/test_rows_centred.py: there sums are
exact.  Digits of q~ beyond the fp32 that it is formed in, the place of a weight's lift,
and keys that are not centred - the start of the products has the rounding that they
would have - move a row by less than its other roundings may: no tolerance made of those
can tell them.)"""
import numpy as np
import pytest

import rows_close
import sparse_exact
from rows_exact import Tokens
from workloads import synth

SHAPES = [(128, 4, 4, 64), (128, 2, 2, 64), (64, 4, 8, 192), (64, 2, 1, 64), (128, 3, 4, 64), (64, 3, 2, 128)]


@pytest.mark.parametrize("name", sorted(set(sparse_exact.STATES) - {"far zeros"}))
@pytest.mark.parametrize("d,bits,G,slots", SHAPES)
def test_a_planted_mistake_is_outside(name, d, bits, G, slots):
    host, q, t, sel, n = state = sparse_exact.state(name, d, bits, G, 2, 3, slots)
    want, s, _, _ = rows_close.weighted(host, q, t, np.zeros((3, 2, host.max_pages)), sel, n)
    assert rows_close.off(want, want, s) == (0.0, 0.0)
    right, _ = sparse_exact.rows(*state)
    assert np.abs(right - want).max() <= 1e-13 * np.abs(want).max()
    wrong, _ = sparse_exact.rows(*state, plant=sparse_exact.STATES[name])
    most, rms = rows_close.off(wrong, want, s)
    assert rms > 1.0, (most, rms)
    # far below an output's size
    assert (s <= 1e-5 * np.linalg.norm(want, axis=-1)).all()


@pytest.mark.parametrize("d,bits,G,slots", SHAPES)
def test_weights_of_one_part_are_outside(d, bits, G, slots):
    host, q, t, _, _ = sparse_exact.state("sums", d, bits, G, 1, 3, slots)
    queries = synth.bf16_bits_to_float(q).astype(np.float64).reshape(3, G, d)
    for b in range(3):
        tok = Tokens(host, b, 0, [(b, i) for i in range(host.every(b))])
        want, s, _, w, _ = rows_close.one(host, queries[b, 0], t[0].astype(np.float64), tok, d ** -0.5)
        m = len(tok.ks)
        p = w / w.max() * 2.0 ** 6
        got = (((p[:m] * tok.vs).astype(np.float16).astype(np.float64)) @ tok.vc + p[:m] @ tok.vz + p[m:] @ tok.vw) / p.sum()
        assert rows_close.off(got[None], want[None], np.array([s]))[0] > 1.0
