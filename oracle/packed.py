"""CPU checker for the operators on packed sequences: attention with grouped heads and scaled embedding, forward and backward.
TEST INFRASTRUCTURE ONLY (see oracle/transformer.py); NumPy float64, one sequence and one head at a time, no blocking.

seq_start[s] .. seq_start[s + 1] - 1 are the rows of sequence s.  Rows in no sequence come out as `untouched` (zero by default).
q: [tokens][h][dh]; k, v: [tokens][h_kv][dh]; head i reads K/V head i // (h // h_kv).  lse: [h][tokens].

Pins (tests/test_oracle_packed.py): the unpacked checker on equal lengths, central finite differences for every gradient, hand-worked
embeddings."""
from __future__ import annotations

import numpy as np


def spans(seq_start):
    return [(int(a), int(b)) for a, b in zip(seq_start[:-1], seq_start[1:]) if b > a]


def scores(q, k, causal):
    """Scaled scores of one head of one sequence, -inf where hidden."""
    s = q @ k.T / np.sqrt(q.shape[-1])
    if causal:
        n = len(q)
        s = np.where(np.arange(n)[None, :] > np.arange(n)[:, None], -np.inf, s)
    return s


def attention(q, k, v, seq_start, causal):
    """(out, lse)"""
    T, h, dh = q.shape
    g = h // k.shape[1]
    out, lse = np.zeros((T, h, dh)), np.zeros((h, T))
    for a, b in spans(seq_start):
        for i in range(h):
            s = scores(q[a:b, i], k[a:b, i // g], causal)
            m = s.max(axis=-1, keepdims=True)
            e = np.exp(s - m)
            total = e.sum(axis=-1, keepdims=True)
            out[a:b, i] = (e / total) @ v[a:b, i // g]
            lse[i, a:b] = (m + np.log(total))[:, 0]
    return out, lse


def attention_backward(q, k, v, out, dout, lse, seq_start, causal):
    """(dq, dk, dv) from the given out and lse."""
    h, dh = q.shape[1:]
    g = h // k.shape[1]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for a, b in spans(seq_start):
        for i in range(h):
            j = i // g
            p = np.exp(scores(q[a:b, i], k[a:b, j], causal) - lse[i, a:b, None])
            do = dout[a:b, i]
            ds = p * (do @ v[a:b, j].T - (do * out[a:b, i]).sum(-1, keepdims=True))
            dq[a:b, i] = ds @ k[a:b, j] / np.sqrt(dh)
            dk[a:b, j] += ds.T @ q[a:b, i] / np.sqrt(dh)
            dv[a:b, j] += p.T @ do
    return dq, dk, dv


def embed(ids, tok, pos, seq_start, scale):
    """pos may be None; ids outside the table and positions behind it contribute zeros."""
    x = np.zeros((len(ids), tok.shape[1]))
    for a, b in spans(seq_start):
        for t in range(a, b):
            if 0 <= ids[t] < len(tok):
                x[t] = scale * tok[ids[t]]
            if pos is not None and t - a < len(pos):
                x[t] += pos[t - a]
    return x


def embed_backward(dx, ids, seq_start, scale, V, S):
    """(dtok, dpos)"""
    dtok, dpos = np.zeros((V, dx.shape[1])), np.zeros((S, dx.shape[1]))
    for a, b in spans(seq_start):
        for t in range(a, b):
            if 0 <= ids[t] < V:
                dtok[ids[t]] += scale * dx[t]
            if t - a < S:
                dpos[t - a] += dx[t]
    return dtok, dpos
