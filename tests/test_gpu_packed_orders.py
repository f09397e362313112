"""Packed attention on batches whose blocks are taken longest first, and with a block's keys in two parts: every row is computed, by whichever
workgroup takes its block, from its own sequence alone."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_packed_attention import Case        # noqa: E402
from test_packed_forms import SHAPES, name, ragged    # noqa: E402


def _case(shape, edit=None):
    n, longest, seed, h, kv, dh, causal = shape
    return Case("bf16", ragged(n, longest, seed), h, kv, dh, causal, first=5, tail=11, seed=n + h, edit=edit)


@pytest.mark.parametrize("shape", SHAPES, ids=name)
def test_scores_far_below_zero(shape):
    """Scores around -450 (d_head 64) and -320: a row that took its reference point from another sequence, or none, would sum to 0."""
    def far(c):
        c.q[:, :, 0], c.k[:, :, 0] = 60, -60
        c.q[:, :, 1:] *= 0.25

    c = _case(shape, far)
    o, lse = c.check_forward()
    assert (lse[:, c.live] < -100).all()
    c.check_backward()


@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] > 1], ids=name)
def test_values_of_other_sequences(shape):
    """NaN and infinities in every fifth sequence: the others come out as they do without them, to the same tolerance."""
    def poison(c):
        for a, b in zip(c.start[1:-1:5], c.start[2::5]):
            for x in (c.q, c.k, c.v, c.do):
                x[a:b:3], x[a + 1:b:3], x[a + 2:b:3] = np.nan, np.inf, -np.inf

    good, bad = _case(shape), _case(shape, poison)
    rows = np.ones(good.T, bool)
    for a, b in zip(good.start[1:-1:5], good.start[2::5]):
        rows[a:b] = False
    good.check_forward(bad.forward(), rows)
    good.check_backward(bad.backward(*good.saved()), rows)
