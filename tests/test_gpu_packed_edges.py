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


# Sequences of which rows see some tiles in part and some as a whole: what a row gets does not depend on which
ODD = KERNELS + [("bf16", [64, 128, 320], 4, 2, 64, 0), ("bf16", [64, 128, 320], 4, 2, 128, 0)]
AT = 20     # a key of every sequence that gets no weight


@pytest.mark.parametrize("dtype,lens,h,kv,dh,shift", ODD, ids=name)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("far", [-np.inf, -1e4])
def test_an_infinite_value_whose_weight_is_zero(dtype, lens, h, kv, dh, shift, causal, far):
    """A key with a score of -inf, or so low that its weight is 0 in 32 bits, with an infinity in V: 0 times it is NaN, in that column of
    the rows that see the key."""
    def edit(c):
        c.q[:, :, 0] = 1
        c.k[:, :, 0] = 0
        c.k[c.start[:-1] + AT, :, 0] = far
        c.v[c.start[:-1] + AT, :, 5] = np.inf

    c = Case(dtype, lens, h, kv, dh, causal, 3, 2, shift=shift, seed=8, edit=edit)
    o, lse = c.forward()
    assert np.isfinite(lse[:, c.live]).all()
    for a, b in zip(c.start[:-1], c.start[1:]):
        first = a + AT if causal else a
        assert np.isnan(o[first:b, :, 5]).all()
        assert np.isfinite(o[a:first]).all() and np.isfinite(np.delete(o[a:b], 5, axis=2)).all()


@pytest.mark.parametrize("dtype,lens,h,kv,dh,shift", ODD, ids=name)
@pytest.mark.parametrize("causal", [False, True])
def test_an_infinite_key_whose_weight_is_zero(dtype, lens, h, kv, dh, shift, causal):
    """A key with an infinity that makes its scores -inf: P and dS are 0, and dQ = dS K is NaN in that column of the rows that see it."""
    def edit(c):
        c.q[:, :, 5] = 1
        c.k[c.start[:-1] + AT, :, 5] = -np.inf

    c = Case(dtype, lens, h, kv, dh, causal, 3, 2, shift=shift, seed=8, edit=edit)
    o, lse = c.forward()
    assert np.isfinite(o[c.live]).all() and np.isfinite(lse[:, c.live]).all()
    dq, dk, dv = c.backward(o, lse)
    for a, b in zip(c.start[:-1], c.start[1:]):
        first = a + AT if causal else a
        assert np.isnan(dq[first:b, :, 5]).all()
        assert np.isfinite(dq[a:first]).all() and np.isfinite(np.delete(dq[a:b], 5, axis=2)).all()
        assert np.isfinite(dk[a:b]).all() and np.isfinite(dv[a:b]).all()


@pytest.mark.parametrize("dtype,lens,h,kv,dh,shift", ODD, ids=name)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinite_gradient_whose_weight_is_zero(dtype, lens, h, kv, dh, shift, causal, sign):
    """An infinity in dO of every sequence's last row: dV = P^T dO is NaN in that column of the key that the row gives no weight, and
    that infinity for all others."""
    def edit(c):
        c.q[:, :, 0] = 1
        c.k[:, :, 0] = 0
        c.k[c.start[:-1] + AT, :, 0] = -np.inf
        c.do[c.start[1:] - 1, :, 5] = sign * np.inf

    c = Case(dtype, lens, h, kv, dh, causal, 3, 2, shift=shift, seed=8, edit=edit)
    o, lse = c.forward()
    dv = c.backward(o, lse)[2]
    for a, b in zip(c.start[:-1], c.start[1:]):
        assert np.isnan(dv[a + AT, :, 5]).all()
        assert (np.delete(dv[a:b, :, 5], AT, axis=0) == sign * np.inf).all()
        assert np.isfinite(np.delete(dv[a:b], 5, axis=2)).all()


def _overlapping(n, T):
    """Every second pair of boundaries is a sequence of all T rows: together far longer than the buffer."""
    return [0, T] * (n // 2) + [0]


@pytest.mark.parametrize("start", [[2 ** 31 - 1, -2 ** 31, 5], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1], [2 ** 31 - 1] * 4, [-2 ** 31] * 4,
                                   _overlapping(300, 100), [5, -2 ** 31, 60, 2 ** 31 - 1]], ids=lambda s: f"{len(s)}from{s[0]}")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embedding_boundaries_at_the_ends_of_32_bits_stay_inside_the_buffers(start, dtype):
    """Undefined results, but what lies around the buffers keeps its values."""
    pf, _ = _mods()
    T, V, S, d, pad, n_seq = 100, 40, 130, 64, 64, len(start) - 1
    tt, code = (torch.bfloat16, pf.PF_DTYPE_BF16) if dtype == "bf16" else (torch.float32, pf.PF_DTYPE_F32)
    gen = torch.Generator(device="cuda").manual_seed(1)
    buf = {n: torch.full((rows + 2 * pad, d), 3.0, device="cuda", dtype=t) for n, rows, t in (("x", T, tt), ("dtok", V, torch.float32), ("dpos", S, torch.float32))}
    at = lambda n: buf[n].data_ptr() + pad * d * buf[n].element_size()
    src = torch.randn(S, d, device="cuda", generator=gen).to(tt)
    ids = torch.arange(T, device="cuda", dtype=torch.int32) % V
    s = torch.tensor(start, dtype=torch.int64).to(torch.int32).cuda()
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.full((n + 256,), 0x7f, dtype=torch.uint8, device="cuda")
    pf.pf_op_embed_packed(code, ids.data_ptr(), src.data_ptr(), src.data_ptr(), s.data_ptr(), n_seq, 1.0, at("x"), T, S, d, V)
    for accumulate in (0, 1):
        pf.pf_op_embed_packed_bwd(code, src.data_ptr(), ids.data_ptr(), s.data_ptr(), n_seq, 1.0, at("dtok"), at("dpos"), accumulate, ws.data_ptr(), n, T, S, d, V)
        torch.cuda.synchronize()
        for t in buf.values():
            assert (t[:pad] == 3.0).all() and (t[-pad:] == 3.0).all()
        assert (ws[n:] == 0x7f).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [24, 520])
def test_embedding_operands_aligned_to_16_bytes_and_no_more(dtype, d):
    """The same bits as from allocations of their own, which are aligned to 256 bytes and more."""
    pf, _ = _mods()
    tt, code = (torch.bfloat16, pf.PF_DTYPE_BF16) if dtype == "bf16" else (torch.float32, pf.PF_DTYPE_F32)
    T, V, S, lens = 150, 37, 90, [90, 1, 40]
    gen = torch.Generator(device="cuda").manual_seed(d)
    normal = lambda n, t: torch.randn(n, d, device="cuda", generator=gen).to(t)
    start = torch.tensor([3] + [3 + sum(lens[:i + 1]) for i in range(3)], device="cuda", dtype=torch.int32)
    ids = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    operands = {"tok": normal(V, tt), "pos": normal(S, tt), "dx": normal(T, tt), "x": torch.zeros(T, d, device="cuda", dtype=tt),
                "dtok": torch.ones(V, d, device="cuda"), "dpos": torch.ones(S, d, device="cuda")}
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    results = []
    for by in (0, 16):
        at = {}
        for k, t in operands.items():
            room = torch.zeros(t.numel() + 64, device="cuda", dtype=t.dtype)
            at[k] = room[by // t.element_size():][:t.numel()].view(t.shape)
            at[k].copy_(t)
            assert at[k].data_ptr() % 32 == by % 32
        p = {k: t.data_ptr() for k, t in at.items()}
        pf.pf_op_embed_packed(code, ids.data_ptr(), p["tok"], p["pos"], start.data_ptr(), 3, 1.5, p["x"], T, S, d, V)
        got = [at["x"].clone()]
        for accumulate in (0, 1):
            pf.pf_op_embed_packed_bwd(code, p["dx"], ids.data_ptr(), start.data_ptr(), 3, 1.5, p["dtok"], p["dpos"], accumulate, ws.data_ptr(), n, T, S, d, V)
            got += [at["dtok"].clone(), at["dpos"].clone()]
        results.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert all(bool(t.any()) for t in results[0])


def test_embedding_of_the_widest_rows():
    """One row of 2^31 - 8 columns: a column's number and the next one's a wave goes on to pass 31 bits.  55 GB."""
    pf, _ = _mods()
    d, V, piece = 2 ** 31 - 8, 1, 1 << 26
    if torch.cuda.mem_get_info()[0] < 70 << 30:
        pytest.skip("needs 70 GB of free device memory")
    gen = torch.Generator(device="cuda").manual_seed(3)
    some = torch.randn(piece, device="cuda", generator=gen).to(torch.bfloat16)
    tok, x = (torch.empty(V * d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for c in range(0, d, piece):
        tok[c:c + piece] = some[:min(piece, d - c)]
    x.fill_(7.0)
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    pf.pf_op_embed_packed(pf.PF_DTYPE_BF16, ids.data_ptr(), tok.data_ptr(), None, None, 0, 1.0, x.data_ptr(), 1, 1, d, V)
    torch.cuda.synchronize()
    same = lambda a, f: all(torch.equal(a[c:c + piece], f(some[:min(piece, d - c)])) for c in range(0, d, piece))
    assert same(x, lambda p: p)
    del tok
    dtok = torch.full((V * d,), 5.0, device="cuda")
    n = pf.pf_op_embed_packed_bwd_workspace(1, 1, d, V)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for accumulate, id_, want in ((0, 0, lambda p: 2.0 * p.float()), (1, 0, lambda p: 4.0 * p.float()), (0, 5, lambda p: torch.zeros_like(p, dtype=torch.float32))):
        ids.fill_(id_)       # 5: no row of the table, which becomes zeros
        pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_BF16, x.data_ptr(), ids.data_ptr(), None, 0, 2.0, dtok.data_ptr(), None, accumulate, ws.data_ptr(), n, 1, 1, d, V)
        torch.cuda.synchronize()
        assert same(dtok, want), (accumulate, id_)


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 32), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_operands_and_gradients_in_buffers_of_their_own(dtype, dh, causal):
    """Q, K and V with a stride each, none of them the other's, no lse asked for: the same bits as from one fused buffer."""
    pf, _ = _mods()
    lens, h, kv = [90, 1, 140], 4, 2
    c = Case(dtype, lens, h, kv, dh, causal, 2, 3, seed=11)
    o, lse = c.forward()
    want = c.backward(o, lse)
    code = pf.PF_DTYPE_F32 if dtype == "f32" else pf.PF_DTYPE_BF16
    lds = [h * dh, kv * dh + 8, kv * dh + 40, h * dh + 16]
    desc = pf.packed_attn(code, c.T, len(lens), h, kv, dh, causal, 0, *lds[1:])     # 0: no gaps

    def put(a, ld, fill=np.nan):
        rows = np.full((c.T, ld), fill, np.float32)
        rows[:, :a.shape[1] * dh] = a.reshape(c.T, -1)
        return torch.from_numpy(rows).cuda().to(torch.float32 if dtype == "f32" else torch.bfloat16)

    q, k, v, do, out = (put(a, ld) for a, ld in ((c.q, lds[0]), (c.k, lds[1]), (c.v, lds[2]), (c.do, lds[3]), (o, lds[3])))
    got = torch.full_like(out, 7.0)
    pf.pf_op_attention_packed(desc, c.d_start.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), got.data_ptr())
    d_lse = torch.from_numpy(lse).cuda()
    grads = [torch.full_like(x, 7.0) for x in (q, k, v)]
    n = pf.pf_op_attention_packed_bwd_workspace(desc)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    pf.pf_op_attention_packed_bwd(desc, c.d_start.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), do.data_ptr(), d_lse.data_ptr(),
                                  *(g.data_ptr() for g in grads), ws.data_ptr(), n)
    torch.cuda.synchronize()
    for x, w in zip([got] + grads, (o,) + want):
        x, heads = x.float().cpu().numpy(), w.shape[1]
        assert np.array_equal(x[c.live, :heads * dh], w.reshape(c.T, -1)[c.live])
        assert (x[~c.live] == 7.0).all() and (x[:, heads * dh:] == 7.0).all()


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 16), ("bf16", 64), ("bf16", 128)])
def test_a_batch_of_empty_sequences(dtype, dh):
    """Nothing is written: the checks of rows that no sequence holds are in forward and backward themselves."""
    c = Case(dtype, [0, 0, 0], 4, 2, dh, True, 37, 20)
    c.forward()
    c.backward(np.zeros((c.T, 4, dh), np.float32), np.zeros((4, c.T), np.float32))


@pytest.mark.parametrize("dtype,dh", [("f32", 8), ("f32", 64), ("bf16", 32), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("n,h,kv", [(1, 65535, 1), (1, 65535, 13107), (5000, 4, 2), (70000, 1, 1)])
def test_sequences_of_one_token_in_closed_form(dtype, dh, n, h, kv):
    """The most heads, and more sequences than a wave looks at at once: out = v, lse = the row's score, dV = the sum of dO over the heads of a
    group, dS = P (dP - D) = 0 up to the rounding of dP - D, at most (d_head + 2) 2^-24 sum |do| (|v| + |out|), and dQ, dK that times scale |k|, |q|."""
    pf, _ = _mods()
    tt, code = (torch.float32, pf.PF_DTYPE_F32) if dtype == "f32" else (torch.bfloat16, pf.PF_DTYPE_BF16)
    gen = torch.Generator(device="cuda").manual_seed(n + h)
    rnd = lambda heads: torch.randn(n, heads, dh, device="cuda", generator=gen).to(tt)
    q, k, v, do = rnd(h), rnd(kv), rnd(kv), rnd(h)
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    desc = pf.packed_attn(code, n, n, h, kv, dh, True)
    out, lse = torch.zeros_like(q), torch.zeros(h, n, device="cuda")
    pf.pf_op_attention_packed(desc, start.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr())
    dq, dk, dv = (torch.full_like(x, 7.0) for x in (q, k, v))
    m = pf.pf_op_attention_packed_bwd_workspace(desc)
    ws = torch.full((m,), 0xff, dtype=torch.uint8, device="cuda")
    pf.pf_op_attention_packed_bwd(desc, start.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), do.data_ptr(), lse.data_ptr(), dq.data_ptr(),
                                  dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), m)
    torch.cuda.synchronize()
    g, u, scale = h // kv, 2.0 ** -24, dh ** -0.5
    step = 2.0 ** -8 if dtype == "bf16" else u
    by_head = lambda x: x.double().repeat_interleave(g, 1)
    by_group = lambda x: x.view(n, kv, g, -1).sum(2)
    assert torch.equal(out, v.repeat_interleave(g, 1))
    s, mag = (q.double() * by_head(k)).sum(-1) * scale, (q.double() * by_head(k)).abs().sum(-1) * scale
    assert ((lse.double().t() - s).abs() <= u * (dh + 4) * mag + 4 * u * s.abs()).all()
    p = 1 + u * ((dh + 4) * mag + 16 + 4 * s.abs())               # P, exp of a rounding error
    r = 2.0 ** -8 if dtype == "bf16" and dh >= 64 else 0.0       # P as an operand
    sums = by_group(do.double().abs())
    assert ((dv.double() - by_group(do.double())).abs() <= (r + u * (g + 32 + (dh + 4) * float(mag.max()) + 4 * float(s.abs().max()))) * sums + step * sums).all()
    e = u * (dh + 2) * 2 * (do.double() * by_head(v)).abs().sum(-1, keepdim=True) * p[..., None] * 2
    assert (dq.double().abs() <= e * scale * by_head(k).abs() * (1 + 2.0 ** -7) + 2.0 ** -95).all()
    assert (dk.double().abs() <= by_group(e * scale * q.double().abs()) * (1 + 2.0 ** -7) + 2.0 ** -95).all()


@pytest.mark.parametrize("dtype,lens,h,kv,dh,shift", ODD, ids=name)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("score", [np.inf, np.nan])
def test_a_score_of_infinity_or_nan(dtype, lens, h, kv, dh, shift, causal, score):
    """The rows that see it have no softmax: NaN in out and lse.  Rows before it (causal) and other sequences' have theirs."""
    def edit(c):
        c.q[:, :, 3] = 1
        c.k[c.start[0:-1:2] + AT, :, 3] = score

    c = Case(dtype, lens, h, kv, dh, causal, 3, 2, shift=shift, seed=12, edit=edit)
    o, lse = c.forward()
    for s, (a, b) in enumerate(zip(c.start[:-1], c.start[1:])):
        first = b if s % 2 else a + AT if causal else a
        assert np.isnan(o[first:b]).all() and np.isnan(lse[:, first:b]).all()
        assert np.isfinite(o[a:first]).all() and np.isfinite(lse[:, a:first]).all()
