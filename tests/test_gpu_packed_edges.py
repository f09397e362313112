"""Attention and embedding on packed sequences at the edges of their contract: rows without a softmax, infinities that a row does see,
boundaries at the ends of 32 bits, operands aligned to no more than the contract asks for, the widest rows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_packed_attention import Case, _mods     # noqa: E402


# (dtype, lengths, heads, K/V heads, d_head, shift): fp32 products of both types (the last two bf16 rows for their alignment), and every
# form of the bf16 kernels
KERNELS = [
    ("f32", [100, 30], 2, 1, 64, 0),
    ("f32", [100, 30], 2, 1, 32, 1),
    ("bf16", [100, 30], 4, 2, 32, 0),
    ("bf16", [100, 30], 2, 1, 64, 3),
    ("bf16", [100, 30], 2, 1, 128, 4),
    ("bf16", [100, 30], 2, 1, 64, 0),
    ("bf16", [100, 30], 2, 1, 128, 0),
    ("bf16", [200] * 20, 12, 12, 128, 0),
    ("bf16", [90, 110] * 30, 8, 8, 64, 0),
    ("bf16", [150, 250] * 10, 8, 8, 64, 0),
    ("bf16", [97] * 26, 8, 8, 128, 0),
]
name = lambda x: f"{len(x)}x{max(x)}" if isinstance(x, list) else str(x)


@pytest.mark.parametrize("dtype,lens,h,kv,dh,shift", KERNELS, ids=name)
@pytest.mark.parametrize("causal", [False, True])
def test_a_row_that_sees_only_minus_infinity(dtype, lens, h, kv, dh, shift, causal):
    """Its log-sum-exp is -inf and it has no softmax: 0 / 0.  Rows of the other sequences keep theirs."""
    def edit(c):
        c.q[:] = 0
        c.q[:, :, 0] = 1
        c.k[:, :, 0] = 0
        c.k[c.start[-2]:c.start[-1], :, 0] = -np.inf

    c = Case(dtype, lens, h, kv, dh, causal, 3, 2, shift=shift, seed=1, edit=edit)
    o, lse = c.forward()
    a, b = c.start[-2:]
    assert (lse[:, a:b] == -np.inf).all()
    assert np.isnan(o[a:b]).all()
    assert np.isfinite(lse[:, 3:a]).all() and np.isfinite(o[3:a]).all()
