"""Embedding on packed sequences and its gradients by sorted tokens, against the float64 checker.

Tolerances: x is one fused product and sum in fp32 (2^-24 of |scale tok| + |pos|) and one rounding (bf16 2^-8 of |x|).  A
gradient row is a sum of n products in fp32: (n + 2) 2^-24 times the sum of their magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as opk          # noqa: E402
from paper_2410_07192_amd import synth    # noqa: E402

U32 = 2.0 ** -24


def _mods():
    from paper_2410_07192_amd import binding as pf
    from paper_2410_07192_amd import device as dev
    return pf, dev


def _setup(dtype, lens, first, tail, ids_of, V, seed):
    rng = np.random.default_rng(seed)
    start = np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)
    T = int(start[-1]) + tail
    ids = np.asarray(ids_of(rng, T), np.int32)
    rnd = lambda *s: synth.round_to_bf16(rng.standard_normal(s)) if dtype == "bf16" else rng.standard_normal(s).astype(np.float32)
    return rng, start, T, ids, rnd


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _code(pf, dtype):
    return pf.PF_DTYPE_BF16 if dtype == "bf16" else pf.PF_DTYPE_F32


uniform = lambda V: lambda rng, T: rng.integers(0, V, T)
frequent = lambda V: lambda rng, T: np.minimum(np.exp(rng.random(T) * np.log(V + 1)).astype(np.int64) - 1, V - 1)
one = lambda rng, T: np.full(T, 3)
outside = lambda V: lambda rng, T: rng.integers(-V, 2 * V, T)
extremes = lambda rng, T: rng.choice([-2 ** 31, -1, 0, 2 ** 31 - 1, 5], T)

# (dtype, lengths, rows before, rows behind, ids, V, S, d, with positions)
CASES = [
    ("bf16", [1], 0, 0, uniform(10), 10, 4, 8, True),
    ("f32", [1], 2, 3, uniform(10), 10, 1, 520, True),
    ("bf16", [5, 0, 130, 1], 3, 40, uniform(300), 300, 130, 768, True),
    ("bf16", [5, 0, 130, 1], 3, 40, outside(300), 300, 100, 64, True),        # ids outside, positions behind the table
    ("f32", [200, 3, 90, 0, 17], 0, 0, frequent(10007), 10007, 256, 512, True),
    ("f32", [33] * 9, 1, 1, extremes, 64, 40, 24, True),
    ("bf16", [1500, 600], 0, 9, one, 5000, 1500, 136, True),                 # one token throughout
    ("bf16", [7] * 300, 0, 0, frequent(2000), 2000, 16, 1032, True),
    ("bf16", [2] * 70 + [0] * 70 + [900] * 5, 4, 0, frequent(50257), 50257, 1024, 256, True),
    ("bf16", [6000], 0, 0, uniform(3), 3, 6000, 72, False),
    ("f32", [400] * 16, 0, 50, frequent(300000), 300000, 400, 8, True),      # more ids than a workgroup's counters times 256
]


@pytest.mark.parametrize("dtype,lens,first,tail,ids_of,V,S,d,with_pos", CASES, ids=[f"{c[0]}-{len(c[1])}x{max(c[1])}-V{c[5]}-d{c[7]}" for c in CASES])
def test_forward_and_backward(dtype, lens, first, tail, ids_of, V, S, d, with_pos):
    pf, _ = _mods()
    rng, start, T, ids, rnd = _setup(dtype, lens, first, tail, ids_of, V, seed=T_seed(lens, V))
    tok, pos, dx = rnd(V, d), rnd(S, d), rnd(T, d)
    live = np.zeros(T, bool)
    live[first:start[-1]] = True
    dx[~live] = np.nan
    scale = 3.25
    d_start, d_ids = torch.from_numpy(start).cuda(), torch.from_numpy(ids).cuda()
    d_tok, d_pos, d_dx = (_dev(a, dtype) for a in (tok, pos, dx))
    x = _dev(np.full((T, d), 7.0), dtype)
    ppos = d_pos.data_ptr() if with_pos else None
    pf.pf_op_embed_packed(_code(pf, dtype), d_ids.data_ptr(), d_tok.data_ptr(), ppos, d_start.data_ptr(), len(lens), scale, x.data_ptr(), T, S, d, V)
    got = x.float().cpu().numpy()
    want = opk.embed(ids, tok.astype(np.float64), pos.astype(np.float64) if with_pos else None, start, scale)
    mag = opk.embed(ids, np.abs(tok).astype(np.float64), np.abs(pos).astype(np.float64) if with_pos else None, start, scale)
    assert (got[~live] == 7.0).all()
    tol = 2 * U32 * mag + (2.0 ** -8 if dtype == "bf16" else U32) * np.abs(want)
    assert (np.abs(got - want)[live] <= tol[live]).all()

    clean = np.where(live[:, None], dx, 0).astype(np.float64)
    wt, wp = opk.embed_backward(clean, ids, start, scale, V, S)
    mt, mp = opk.embed_backward(np.abs(clean), ids, start, scale, V, S)
    nt, npos = opk.embed_backward(np.ones((T, 1)), ids, start, 1.0, V, S)
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    for accumulate in (0, 1):
        dtok = torch.full((V + 1, d), 5.0, device="cuda")
        dpos = torch.full((S + 1, d), -2.0, device="cuda")
        for again in range(2):
            ws = torch.full((n,), 0xff if again else 0, dtype=torch.uint8, device="cuda")
            g = dtok.clone(), dpos.clone()
            pf.pf_op_embed_packed_bwd(_code(pf, dtype), d_dx.data_ptr(), d_ids.data_ptr(), d_start.data_ptr(), len(lens), scale, g[0].data_ptr(),
                                      g[1].data_ptr() if with_pos else None, accumulate, ws.data_ptr(), n, T, S, d, V)
            a = [t.cpu().numpy() for t in g]
            if again:
                assert np.array_equal(a[0], before[0]) and np.array_equal(a[1], before[1])      # bit for bit
            before = a
        assert (a[0][V] == 5.0).all() and (a[1][S] == -2.0).all()
        for name, x_, w, m, cnt, base in (("dtok", a[0][:V], wt, mt, nt, 5.0), ("dpos", a[1][:S], wp, mp, npos, -2.0)):
            if name == "dpos" and not with_pos:
                assert (x_ == -2.0).all()
                continue
            add = base if accumulate else 0.0
            tol = (cnt + 2) * U32 * m + 2 * U32 * abs(add)
            err = np.abs(x_ - (w + add))
            assert (err <= tol).all(), (name, accumulate, (err - tol).max())


def T_seed(lens, V):
    return sum(lens) + V


def test_one_sequence_without_boundaries():
    pf, _ = _mods()
    T, V, S, d = 300, 50, 256, 64
    rng, start, T, ids, rnd = _setup("f32", [T], 0, 0, uniform(V), V, 1)
    tok, pos, dx = (torch.from_numpy(rnd(n, d)).cuda() for n in (V, S, T))
    d_ids = torch.from_numpy(ids).cuda()
    ws = torch.empty(pf.pf_op_embed_packed_bwd_workspace(T, S, d, V), dtype=torch.uint8, device="cuda")
    res = []
    for s, n in ((torch.from_numpy(start).cuda(), 1), (None, 0)):
        p = s.data_ptr() if s is not None else None
        x, dtok, dpos = torch.zeros(T, d, device="cuda"), torch.zeros(V, d, device="cuda"), torch.zeros(S, d, device="cuda")
        pf.pf_op_embed_packed(pf.PF_DTYPE_F32, d_ids.data_ptr(), tok.data_ptr(), pos.data_ptr(), p, n, 2.0, x.data_ptr(), T, S, d, V)
        pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_F32, dx.data_ptr(), d_ids.data_ptr(), p, n, 2.0, dtok.data_ptr(), dpos.data_ptr(), 0, ws.data_ptr(),
                                  ws.numel(), T, S, d, V)
        res.append([t.cpu() for t in (x, dtok, dpos)])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_captured_with_other_tokens():
    pf, _ = _mods()
    V, S, d, T, n_seq = 997, 64, 264, 1000, 20
    gen = torch.Generator(device="cuda").manual_seed(2)
    dx = torch.randn(T, d, device="cuda", generator=gen).to(torch.bfloat16)
    tok, pos = torch.randn(V, d, device="cuda", generator=gen).to(torch.bfloat16), torch.randn(S, d, device="cuda", generator=gen).to(torch.bfloat16)
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    start = torch.linspace(0, T, n_seq + 1, device="cuda").to(torch.int32)
    x, dtok, dpos = torch.zeros(T, d, device="cuda", dtype=torch.bfloat16), torch.zeros(V, d, device="cuda"), torch.zeros(S, d, device="cuda")
    ws = torch.empty(pf.pf_op_embed_packed_bwd_workspace(T, S, d, V), dtype=torch.uint8, device="cuda")

    def call():
        st = torch.cuda.current_stream().cuda_stream
        pf.pf_op_embed_packed(pf.PF_DTYPE_BF16, ids.data_ptr(), tok.data_ptr(), pos.data_ptr(), start.data_ptr(), n_seq, 1.5, x.data_ptr(), T, S, d, V, st)
        pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_BF16, dx.data_ptr(), ids.data_ptr(), start.data_ptr(), n_seq, 1.5, dtok.data_ptr(), dpos.data_ptr(), 0,
                                  ws.data_ptr(), ws.numel(), T, S, d, V, st)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        ids.copy_(torch.randint(0, 3 if turn == 2 else V, (T,), device="cuda", generator=gen, dtype=torch.int32))
        if turn == 3:
            start.copy_(torch.arange(n_seq + 1, device="cuda").to(torch.int32) * 3 + 2)
        results = (x, dtok, dpos)
        for t in results:
            t.fill_(1.0)
        call()
        want = [t.clone() for t in results]
        for t in results:
            t.fill_(1.0)
        ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), turn


@pytest.mark.parametrize("start", [[50, 10, 90], [-5, 20, 1000], [100, 100, 100], [0, 0, 0], [7, -3, -9]])
def test_boundaries_out_of_order_or_range_stay_inside_the_buffers(start):
    """Undefined results, but rows around the buffers keep their values."""
    pf, _ = _mods()
    T, V, S, d = 100, 40, 30, 64
    pad = 64
    buf = {n: torch.full(((rows + 2 * pad), d), 3.0, device="cuda") for n, rows in (("x", T), ("dtok", V), ("dpos", S))}
    at = lambda n: buf[n].data_ptr() + pad * d * 4
    src = torch.randn(T, d, device="cuda")
    ids = torch.arange(T, device="cuda", dtype=torch.int32) % V
    s = torch.tensor(start, dtype=torch.int32, device="cuda")
    n = pf.pf_op_embed_packed_bwd_workspace(T, S, d, V)
    ws = torch.full((n + 256,), 0x7f, dtype=torch.uint8, device="cuda")
    pf.pf_op_embed_packed(pf.PF_DTYPE_F32, ids.data_ptr(), src.data_ptr(), src.data_ptr(), s.data_ptr(), 2, 1.0, at("x"), T, S, d, V)
    pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_F32, src.data_ptr(), ids.data_ptr(), s.data_ptr(), 2, 1.0, at("dtok"), at("dpos"), 0, ws.data_ptr(), n, T, S, d, V)
    torch.cuda.synchronize()
    for t in buf.values():
        assert (t[:pad] == 3.0).all() and (t[-pad:] == 3.0).all()
    assert (ws[n:] == 0x7f).all()
