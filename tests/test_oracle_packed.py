"""Pins of the packed checker: the unpacked one on equal lengths, finite differences, hand-worked embeddings."""
import numpy as np
import pytest

from oracle import packed as opk
from oracle import transformer as ot


@pytest.mark.parametrize("causal", [False, True])
def test_equal_lengths_and_heads_match_the_unpacked_checker(causal):
    rng = np.random.default_rng(0)
    B, S, h, dh = 3, 7, 2, 8
    q, k, v = (rng.standard_normal((B * S, h, dh)) for _ in range(3))
    out, _ = opk.attention(q, k, v, np.arange(B + 1) * S, causal)
    heads = lambda x: x.reshape(B, S, h, dh).transpose(0, 2, 1, 3)
    want = ot.attention_probs(heads(q), heads(k), causal) @ heads(v)
    assert np.allclose(heads(out), want, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_by_finite_differences(causal):
    rng = np.random.default_rng(1)
    start = np.array([1, 4, 4, 9])
    T, h, kv, dh = 11, 4, 2, 3
    q, w = rng.standard_normal((T, h, dh)), rng.standard_normal((T, h, dh))
    k, v = rng.standard_normal((T, kv, dh)), rng.standard_normal((T, kv, dh))
    loss = lambda: float((opk.attention(q, k, v, start, causal)[0] * w).sum())
    out, lse = opk.attention(q, k, v, start, causal)
    grads = opk.attention_backward(q, k, v, out, w, lse, start, causal)
    for x, g in zip((q, k, v), grads):
        for at in [tuple(rng.integers(0, n) for n in x.shape) for _ in range(25)]:
            keep = x[at]
            x[at] = keep + 1e-5
            up = loss()
            x[at] = keep - 1e-5
            down = loss()
            x[at] = keep
            assert abs((up - down) / 2e-5 - g[at]) < 1e-7
    assert not grads[0][0].any() and not grads[1][9:].any()        # rows in no sequence


def test_embedding_hand_worked():
    tok = np.array([[1.0, 2.0], [10.0, 20.0], [100.0, 200.0]])
    pos = np.array([[0.5, 0.25], [0.125, 0.0625]])
    ids = np.array([9, 1, 2, 0, 3, 1])
    start = np.array([1, 4, 4, 6])                                  # rows 1-3 and 4-5
    x = opk.embed(ids, tok, pos, start, 2.0)
    assert x.tolist() == [[0, 0], [20.5, 40.25], [200.125, 400.0625], [2, 4], [0.5, 0.25], [20.125, 40.0625]]
    dx = np.arange(12.0).reshape(6, 2)
    dtok, dpos = opk.embed_backward(dx, ids, start, 2.0, 3, 2)
    assert dtok.tolist() == [[12, 14], [24, 28], [8, 10]]
    assert dpos.tolist() == [[10, 12], [14, 16]]
