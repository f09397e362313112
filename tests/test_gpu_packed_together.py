"""The operators on packed sequences as they are used: one layer forward and backward through them and the library's other operators,
gradients against differences, every form of the bf16 kernels, and calls side by side."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as opk                                # noqa: E402
from paper_2410_07192_amd import synth                          # noqa: E402
from test_gpu_packed_attention import Case, U16, U32, _mods     # noqa: E402


# Lengths, heads, K/V heads, d_head, causal.  With the sizes of test_gpu_packed_attention these reach every form of the forward (tiles
# shared by the waves of a workgroup, keys in one or two parts; independent waves, 1, 2 or 4 to a block) for both d_head, and the
# backward in one part and several.
FORMS = [
    ([200] * 20, 12, 12, 128, True),                # shared tiles
    ([2000], 12, 12, 128, False),                   # shared tiles in two parts
    ([90, 110] * 30, 8, 8, 64, False),              # one wave
    ([150, 250] * 10, 8, 8, 64, True),              # two waves
    ([40, 300, 1, 120] * 10, 8, 2, 128, True),
    ([700, 900], 16, 16, 64, False),
    ([2400], 16, 2, 128, False),
    ([1] * 190, 48, 16, 128, True),                 # one wave, d_head 128
    ([60] * 12, 48, 16, 128, True),
    ([3] * 51, 36, 12, 128, False),                 # two waves
    ([323], 48, 12, 128, False),                    # shared tiles in two parts
    ([33, 40] * 20, 24, 8, 64, False),              # one wave, d_head 64
]


@pytest.mark.parametrize("lens,h,kv,dh,causal", FORMS, ids=lambda x: "x".join(map(str, x[:2])) if isinstance(x, list) else str(x))
def test_forms(lens, h, kv, dh, causal):
    c = Case("bf16", lens, h, kv, dh, causal, first=5, tail=11, seed=h)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_sequences_that_begin_where_a_tile_ends(dtype, dh, causal):
    """Tiles that rows of one sequence see all of and rows of the next nothing of, with scores around -400: a sequence whose softmax
    took its reference point from another's tiles, or none, would sum to 0."""
    def far(c):
        c.q[:, :, 0], c.k[:, :, 0] = 60, -60
        c.q[:, :, 1:] *= 0.25

    c = Case(dtype, [64, 128, 70, 192, 64, 1, 63, 320], 4, 2, dh, causal, first=5, tail=3, seed=dh, edit=far)
    o, lse = c.check_forward()
    assert (lse[:, c.live] < -100).all()
    c.check_backward()


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_against_differences(causal):
    """f = sum(dout * out) along a direction of each operand, in fp32.  The difference quotient's own error is the 64-bit checker's at
    the same step; on top of it comes the rounding of out (relative error of a probability fp, as in test_gpu_packed_attention)
    over the step, and that of the gradient, at most c times the sums of its terms' magnitudes."""
    lens, h, kv, dh, eps = [37, 1, 20], 4, 2, 32, 2.0 ** -5
    base = Case("f32", lens, h, kv, dh, causal, seed=21)
    rng = np.random.default_rng(22)
    q, k, v, do = base.wide()
    out, lse = opk.attention(q, k, v, base.start, causal)
    g64 = opk.attention_backward(q, k, v, out, do, lse, base.start, causal)
    o32, l32 = base.forward()
    got = base.backward(o32, l32)
    n, grp = max(lens), h // kv
    top = max((np.abs(q[a:b, i]) @ np.abs(k[a:b, i // grp]).T).max() for a, b in opk.spans(base.start) for i in range(h)) / np.sqrt(dh) * (1 + 4 * eps) ** 2
    fp = U32 * ((dh + 4) * top + n + 16)
    c = U32 * ((dh + 4) * top + n * grp + 16 + 4 * np.abs(lse).max() + 2 * (dh + 2))
    absd = [np.abs(x) for x in (q, k, v, do)]
    mags = [np.zeros_like(x) for x in (q, k, v)]
    out_mag = np.zeros_like(out)
    for a, b in opk.spans(base.start):
        for i in range(h):
            j = i // grp
            p = np.exp(opk.scores(q[a:b, i], k[a:b, j], causal) - lse[i, a:b, None])
            w = p * (absd[3][a:b, i] @ absd[2][a:b, j].T + (absd[3][a:b, i] * np.abs(out[a:b, i])).sum(-1, keepdims=True))
            mags[0][a:b, i] = w @ absd[1][a:b, j] / np.sqrt(dh)
            mags[1][a:b, j] += w.T @ absd[0][a:b, i] / np.sqrt(dh)
            mags[2][a:b, j] += p.T @ absd[3][a:b, i]
            out_mag[a:b, i] = absd[2][a:b, j].max(axis=0) * (1 + eps)
    for which in range(3):
        d = rng.choice([-1.0, 1.0], (q, k, v)[which].shape) * (2.0 ** -3)
        f32, f64 = [], []
        for sign in (1, -1):
            moved = [q, k, v]
            moved[which] = (moved[which] + sign * eps * d).astype(np.float32).astype(np.float64)
            edit = lambda cs, m=moved: [setattr(cs, name, x.astype(np.float32)) for name, x in zip("qkv", m)]
            o, _ = Case("f32", lens, h, kv, dh, causal, seed=21, edit=edit).forward()
            f32.append((o.astype(np.float64) * do).sum())
            f64.append((opk.attention(*moved, base.start, causal)[0] * do).sum())
        quotient, exact = (f32[0] - f32[1]) / (2 * eps), (f64[0] - f64[1]) / (2 * eps)
        slope, slope64 = (got[which] * d).sum(), (g64[which] * d).sum()
        tol = abs(exact - slope64) + (absd[3] * (2 * fp + U32) * out_mag).sum() / eps + (np.abs(d) * (c + U32) * mags[which]).sum()
        assert abs(quotient - slope) <= tol, (which, quotient, slope, tol)
        assert tol < 0.2 * np.abs(got[which] * d).sum()      # the bound says something


def test_embedding_gradients_against_differences():
    """x is linear in both tables: the quotient is exact up to the rounding of x (2^-24 of each of its two terms and of itself)."""
    pf, _ = _mods()
    rng = np.random.default_rng(3)
    start = np.array([2, 40, 40, 95], np.int32)
    T, V, S, d, scale, eps = 99, 30, 64, 40, 2.5, 0.5
    ids = rng.integers(0, V, T).astype(np.int32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    tok, pos, dx = (rng.standard_normal(s).astype(np.float32) for s in ((V, d), (S, d), (T, d)))
    d_ids, d_start, d_dx = dev(ids), dev(start), dev(dx)
    live = slice(start[0], start[-1])

    def f(tok, pos):
        x, a, b = torch.zeros(T, d, device="cuda"), dev(tok), dev(pos)
        pf.pf_op_embed_packed(pf.PF_DTYPE_F32, d_ids.data_ptr(), a.data_ptr(), b.data_ptr(), d_start.data_ptr(), 3, scale, x.data_ptr(), T, S, d, V)
        return (x.cpu().numpy().astype(np.float64) * dx)[live].sum()

    dtok, dpos = torch.zeros(V, d, device="cuda"), torch.zeros(S, d, device="cuda")
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_F32, d_dx.data_ptr(), d_ids.data_ptr(), d_start.data_ptr(), 3, scale, dtok.data_ptr(), dpos.data_ptr(), 0,
                              ws.data_ptr(), n, T, S, d, V)
    for which, (table, grad) in enumerate(((tok, dtok), (pos, dpos))):
        step = rng.choice([-1.0, 1.0], table.shape).astype(np.float32)
        up, down = [tok, pos], [tok, pos]
        up[which], down[which] = table + np.float32(eps) * step, table - np.float32(eps) * step
        quotient = (f(*up) - f(*down)) / (2 * eps)
        slope = (grad.cpu().numpy().astype(np.float64) * step).sum()
        mag = scale * (np.abs(tok).max() + eps) + np.abs(pos).max() + eps
        tol = np.abs(dx[live]).sum() * (3 * U32 * mag + scale * U32 * np.abs(table).max()) / eps + (T + 2) * U32 * scale * np.abs(dx[live]).sum()
        assert abs(quotient - slope) <= tol, (which, quotient, slope, tol)


@pytest.mark.parametrize("dtype,dh", [("f32", 32), ("bf16", 64), ("bf16", 128)])
def test_a_layer_on_a_packed_batch(dtype, dh):
    """y = attention(layernorm(x) Wqkv^T) Wo^T + x with x = scale tok[ids] + pos, in a buffer with rows behind the last sequence, and the
    gradients of sum(dy * y) back to both tables and Wqkv, against autograd in 64 bits.

    Tolerance, relative in the Frobenius norm.  fp32: every stage is off by 2^-24 times the terms of its sums; layer norm 2 d, the
    projections d and h dh, scores dh, sums over keys 130, together under 1000 each way, times 4 for the stages' gains.  bf16: eleven
    stored or rounded stages (x, h, qkv, P, a, y; da, dS, dqkv, dh, dx), each off by 2^-8 at most, times 2."""
    pf, _ = _mods()
    T, V, S, d, h, kv, causal, scale = 320, 50, 128, 128, 4, 2, True, 1.5
    lens, eps = [100, 0, 1, 128, 33], 1e-5
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    live, rng = int(start[-1]), np.random.default_rng(dh)
    n_qkv = (h + 2 * kv) * dh
    rnd = lambda *s, scale=1.0: synth.round_to_bf16(rng.standard_normal(s) * scale) if dtype == "bf16" else (rng.standard_normal(s) * scale).astype(np.float32)
    tok, pos, wqkv, wo, dy = rnd(V, d), rnd(S, d), rnd(n_qkv, d, scale=d ** -0.5), rnd(d, h * dh, scale=(h * dh) ** -0.5), rnd(T, d)
    gain, bias = rnd(d, scale=0.1) + np.float32(1), rnd(d, scale=0.1)
    if dtype == "bf16":
        gain = synth.round_to_bf16(gain)
    dy[live:] = 0
    ids = rng.integers(0, V, T).astype(np.int32)

    # the checker
    t64 = lambda a, grad=False: torch.from_numpy(a.astype(np.float64)).requires_grad_(grad)
    p_tok, p_pos, p_wqkv = t64(tok, True), t64(pos, True), t64(wqkv, True)
    at = torch.cat([torch.arange(n) for n in lens])
    x = scale * p_tok[torch.from_numpy(ids[:live]).long()] + p_pos[at]
    xn = torch.nn.functional.layer_norm(x, (d,), t64(gain), t64(bias), eps)
    qkv = xn @ p_wqkv.T
    heads = []
    for a, b in opk.spans(start):
        n = b - a
        q, k, v = (t.reshape(n, -1, dh).transpose(0, 1) for t in qkv[a:b].split([h * dh, kv * dh, kv * dh], 1))
        s = q @ k.repeat_interleave(h // kv, 0).transpose(1, 2) / dh ** 0.5
        s = s.masked_fill(torch.triu(torch.ones(n, n, dtype=torch.bool), 1), -np.inf)
        heads.append((s.softmax(-1) @ v.repeat_interleave(h // kv, 0)).transpose(0, 1).reshape(n, h * dh))
    y64 = torch.cat(heads) @ t64(wo).T + x
    (y64 * t64(dy)[:live]).sum().backward()

    # the operators
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    code = pf.PF_DTYPE_BF16 if dtype == "bf16" else pf.PF_DTYPE_F32
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(tt)
    new = lambda *s: torch.zeros(*s, dtype=tt, device="cuda")
    f32 = lambda *s: torch.zeros(*s, device="cuda")
    P = lambda t, col=0: t.data_ptr() + col * t.element_size()
    d_start, d_ids = torch.from_numpy(start).cuda(), torch.from_numpy(ids).cuda()
    d_tok, d_pos, d_w, d_wo, d_dy, d_g, d_b = (dev(a) for a in (tok, pos, wqkv, wo, dy, gain, bias))
    w_t, wo_t = dev(wqkv.T), dev(wo.T)
    x, xn, qkv, a, y, mean, rstd, lse = new(T, d), new(T, d), new(T, n_qkv), new(T, h * dh), new(T, d), f32(T), f32(T), f32(h, T)
    da, dqkv, dxn, dx, dtok, dpos, dg, db, part = new(T, h * dh), new(T, n_qkv), new(T, d), new(T, d), f32(V, d), f32(S, d), f32(d), f32(d), f32(512 * 2 * d)
    dw = f32(n_qkv, d)
    desc = pf.packed_attn(code, T, len(lens), h, kv, dh, causal, n_qkv, n_qkv, n_qkv)
    n1, n2 = pf.pf_op_attention_packed_bwd_workspace(desc), pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.empty(max(n1, n2), dtype=torch.uint8, device="cuda")    # one after the other on one stream: they may share it

    def step():
        st = torch.cuda.current_stream().cuda_stream
        pf.pf_op_embed_packed(code, P(d_ids), P(d_tok), P(d_pos), P(d_start), len(lens), scale, P(x), T, S, d, V, st)
        pf.pf_op_layernorm(code, P(x), P(d_g), P(d_b), P(xn), T, d, eps, P(mean), P(rstd), st)
        pf.pf_op_gemm(code, P(xn), P(d_w), P(qkv), T, n_qkv, d, stream=st)
        pf.pf_op_attention_packed(desc, P(d_start), P(qkv), P(qkv, h * dh), P(qkv, (h + kv) * dh), P(a), P(lse), st)
        pf.pf_op_gemm(code, P(a), P(d_wo), P(y), T, d, h * dh, resid=P(x), stream=st)
        pf.pf_op_gemm(code, P(d_dy), P(wo_t), P(da), T, h * dh, d, stream=st)
        pf.pf_op_attention_packed_bwd(desc, P(d_start), P(qkv), P(qkv, h * dh), P(qkv, (h + kv) * dh), P(a), P(da), P(lse), P(dqkv), P(dqkv, h * dh),
                                      P(dqkv, (h + kv) * dh), P(ws), n1, st)
        pf.pf_op_gemm(code, P(dqkv), P(w_t), P(dxn), T, d, n_qkv, stream=st)
        if dtype == "bf16":
            dw.zero_()
            pf.pf_op_gemm_tn(code, P(dqkv), P(xn), P(dw), n_qkv, d, T, stream=st)
        pf.pf_op_layernorm_bwd(code, P(dxn), P(x), P(d_g), P(mean), P(rstd), P(d_dy), P(dx), P(dg), P(db), P(part), T, d, st)
        pf.pf_op_embed_packed_bwd(code, P(dx), P(d_ids), P(d_start), len(lens), scale, P(dtok), P(dpos), 0, P(ws), n2, T, S, d, V, st)

    def check():
        torch.cuda.synchronize()
        tol = 4 * 2000 * U32 if dtype == "f32" else 2 * 11 * U16
        pairs = [("y", y[:live], y64), ("dtok", dtok, p_tok.grad), ("dpos", dpos, p_pos.grad)] + ([("dw", dw, p_wqkv.grad)] if dtype == "bf16" else [])
        for name, got, want in pairs:
            want = want.detach()
            err = float((got.double().cpu() - want).norm() / want.norm())
            assert err <= tol, (name, err, tol)

    step()
    check()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (x, xn, qkv, a, y, da, dqkv, dxn, dx, dtok, dpos, dw):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        check()


def test_calls_side_by_side():
    """Two streams, and two graphs on them, each with a workspace of its own; two graphs on one stream that share a workspace."""
    pf, _ = _mods()
    cs = [Case("bf16", [400, 33, 270], 8, 2, 64, True, seed=4), Case("bf16", [130, 500], 8, 2, 128, False, seed=5)]
    want = []
    for c in cs:
        saved = c.saved()
        want.append(c.backward(*saved))
    outs = [c.put(c.saved()[0].reshape(c.T, -1)) for c in cs]
    lses = [torch.from_numpy(c.saved()[1]).cuda() for c in cs]
    dos = [c.put(c.do.reshape(c.T, -1)) for c in cs]
    gs = [c.put(np.full((c.T, c.ld), 7.0)) for c in cs]
    ns = [pf.pf_op_attention_packed_bwd_workspace(c.desc) for c in cs]
    own = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in ns]
    shared = torch.full((max(ns),), 0xff, dtype=torch.uint8, device="cuda")

    def call(i, ws, stream):
        c = cs[i]
        pf.pf_op_attention_packed_bwd(c.desc, c.d_start.data_ptr(), *c.parts(c.qkv), c.at(outs[i]), c.at(dos[i]), lses[i].data_ptr(), *c.parts(gs[i]),
                                      ws.data_ptr(), ns[i], stream)

    def check():
        torch.cuda.synchronize()
        for c, g, w in zip(cs, gs, want):
            got = c.rows(g, c.ld)[:, :(c.h + 2 * c.kv) * c.dh]
            assert np.array_equal(got, np.concatenate([x.reshape(c.T, -1) for x in w], 1), equal_nan=True)
            g.fill_(7.0)
        torch.cuda.synchronize()

    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            call(i, own[i], s.cuda_stream)
    check()
    graphs = {}
    for i in range(2):
        for name, ws in (("own", own[i]), ("shared", shared)):
            graphs[name, i] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[name, i], stream=streams[i]):
                call(i, ws, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for _ in range(3):
        for g in gs:
            g.fill_(7.0)
        torch.cuda.synchronize()
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                graphs["own", i].replay()
        check()
        for i in (0, 1, 1, 0):
            graphs["shared", i].replay()
        check()


@pytest.mark.parametrize("start", [[50, 10, 90], [-5, 20, 1000], [100, 100, 100], [0, 0, 0], [7, -3, -9], [2 ** 31 - 1, -2 ** 31, 5]])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_boundaries_out_of_order_or_range_stay_inside_the_buffers(start, dtype, dh):
    """Undefined results, but what lies around them keeps its values."""
    pf, _ = _mods()
    T, h, kv, pad = 100, 4, 2, 64
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(1)
    width = (h + 2 * kv) * dh
    qkv, do = (torch.randn(T, w, device="cuda", generator=gen).to(tt) for w in (width, h * dh))
    buf = lambda w, t=tt: torch.full((T + 2 * pad, w), 3.0, device="cuda", dtype=t)
    out, g, lse = buf(h * dh), buf(width), torch.full((h * T + 2 * pad,), 3.0, device="cuda")
    es = out.element_size()
    s = torch.tensor(start, dtype=torch.int32, device="cuda")
    for causal in (False, True):
        desc = pf.packed_attn(pf.PF_DTYPE_BF16 if dtype == "bf16" else pf.PF_DTYPE_F32, T, 2, h, kv, dh, causal, width, width, width)
        n = pf.pf_op_attention_packed_bwd_workspace(desc)
        ws = torch.full((n + 256,), 0x7f, dtype=torch.uint8, device="cuda")
        o, l = out.data_ptr() + pad * h * dh * es, lse.data_ptr() + pad * 4
        parts = lambda p: [p + c * dh * es for c in (0, h, h + kv)]
        pf.pf_op_attention_packed(desc, s.data_ptr(), *parts(qkv.data_ptr()), o, l)
        pf.pf_op_attention_packed_bwd(desc, s.data_ptr(), *parts(qkv.data_ptr()), o, do.data_ptr(), l, *parts(g.data_ptr() + pad * width * es), ws.data_ptr(), n)
        torch.cuda.synchronize()
        for t in (out, g):
            assert (t[:pad] == 3.0).all() and (t[-pad:] == 3.0).all()
        assert (lse[:pad] == 3.0).all() and (lse[-pad:] == 3.0).all() and (ws[n:] == 0x7f).all()


@pytest.mark.parametrize("dtype,h,kv,dh,lens", [("bf16", 2, 1, 64, [300, 90, 129]), ("bf16", 2, 1, 128, [300, 90, 129]), ("f32", 2, 1, 64, [300, 90]),
                                                ("bf16", 12, 12, 128, [200] * 20), ("bf16", 8, 8, 64, [90, 110] * 30), ("bf16", 8, 8, 64, [150, 250] * 10)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("none", [64, 70, 128])
def test_scores_of_minus_infinity_before_any_other(dtype, h, kv, dh, lens, causal, none):
    """The first keys of every sequence score -inf: they have probability 0, and the softmax takes its maximum from those that follow, near
    0 or far below.  P and the result are rounded (2^-8 each for bf16), the exponentials and sums of at most 300 keys by 300 2^-24."""
    def edit(c):
        c.q[:] = 0
        c.q[:, :, 0] = 1
        c.k[:, :, 0] = -np.abs(c.k[:, :, 0])
        for i, (a, b) in enumerate(zip(c.start[:-1], c.start[1:])):
            c.k[a:b, :, 0] -= 2000 * (i % 2)
            c.k[a:min(a + none, b), :, 0] = -np.inf

    c = Case(dtype, lens, h, kv, dh, causal, first=3, seed=7, edit=edit)
    o, lse = c.forward()
    r = (2 * U16 if dtype == "bf16" else 0) + 300 * U32 + 1e-5
    for a, b in list(opk.spans(c.start))[:4]:
        s = c.k[a:b, :, 0].astype(np.float64) / np.sqrt(dh)
        for i in range(h):
            j = i // (h // kv)
            for row in range(none, b - a, 17):
                x, v = (s[:row + 1, j], c.v[a:a + row + 1, j]) if causal else (s[:, j], c.v[a:b, j])
                top = x.max()
                p = np.exp(x - top)
                want, mag = (p @ v) / p.sum(), (p @ np.abs(v)) / p.sum()
                assert (np.abs(o[a + row, i] - want) <= r * mag).all(), (a, i, row)
                assert abs(lse[i, a + row] - (top + np.log(p.sum()))) <= 1e-5 + 4 * U32 * abs(top), (a, i, row)


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("V,d,dtype", [(33001, 520, "f32"), (70000, 256, "bf16")])
def test_embedding_gradient_of_a_large_table(V, d, dtype, accumulate):
    """A table of more than 64 MB, whose last rows are cleared in another launch than the first: rows that tokens use and rows that none
    does, in both parts and at the border.  A row's error: its number of terms times 2^-24 of their magnitudes."""
    pf, _ = _mods()
    gen = torch.Generator(device="cuda").manual_seed(V)
    border = V - V // 2
    T, S, scale, lens = 700, 600, 1.5, [600, 3, 90]
    ids = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    ids[5:9], ids[9:60], ids[60:64] = border - 1, border, V - 1
    ids[64:70] = 0
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dx = torch.randn(T, d, device="cuda", generator=gen).to(tt)
    start = torch.tensor([2] + [2 + sum(lens[:i + 1]) for i in range(3)], device="cuda", dtype=torch.int32)
    live = slice(2, 2 + sum(lens))
    dtok, dpos = torch.full((V + 1, d), 0.5, device="cuda"), torch.full((S, d), 0.5, device="cuda")
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_BF16 if dtype == "bf16" else pf.PF_DTYPE_F32, dx.data_ptr(), ids.data_ptr(), start.data_ptr(), 3, scale,
                              dtok.data_ptr(), dpos.data_ptr(), accumulate, ws.data_ptr(), n, T, S, d, V)
    x, at = dx[live].double(), ids[live].long()
    want, mag, count = (torch.zeros(V, w, device="cuda", dtype=torch.double) for w in (d, d, 1))
    want.index_add_(0, at, x * scale)
    mag.index_add_(0, at, x.abs() * scale)
    count.index_add_(0, at, torch.ones(len(at), 1, device="cuda", dtype=torch.double))
    want += 0.5 * accumulate
    torch.cuda.synchronize()
    assert (dtok[V] == 0.5).all()
    assert ((dtok[:V].double() - want).abs() <= (count + 2) * U32 * mag + U32 * accumulate * (count > 0)).all()


@pytest.mark.parametrize("lens,h,kv,dh,causal", [f for f in FORMS if len(f[0]) > 1], ids=lambda x: "x".join(map(str, x[:2])) if isinstance(x, list) else str(x))
def test_values_of_other_sequences_in_every_form(lens, h, kv, dh, causal):
    """NaN and infinities in every fifth sequence: the others come out as they do without them, to the same tolerance."""
    def poison(c):
        for a, b in zip(c.start[1:-1:5], c.start[2::5]):
            for x in (c.q, c.k, c.v, c.do):
                x[a:b:3], x[a + 1:b:3], x[a + 2:b:3] = np.nan, np.inf, -np.inf

    good, bad = (Case("bf16", lens, h, kv, dh, causal, first=5, tail=11, seed=h, edit=e) for e in (None, poison))
    rows = np.ones(good.T, bool)
    for a, b in zip(good.start[1:-1:5], good.start[2::5]):
        rows[a:b] = False
    good.check_forward(bad.forward(), rows)
    good.check_backward(bad.backward(*good.saved()), rows)
