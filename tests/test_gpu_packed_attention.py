"""Attention on packed sequences, forward and backward, against the float64 checker.

Tolerances, element by element.  A product accumulated in fp32 over n terms is off by at most n 2^-24 times the sum of its
terms' magnitudes; an argument x of the exponential by |x| 2^-23.  With top = max over pairs of scale sum |q||k|, the relative
error of a probability is at most fp(n) = 2^-24 ((dh + 4) top + n + 16) against a sum over n keys.  bf16 storage rounds the
result (2^-8 of it), and the bf16 products (d_head 64 and 128) round P and dS (2^-8 of each):
  out   (r + 2 fp) sum P |v|                                     + 2^-8 |out|
  dv    (r + fp) sum P |do|                                      + 2^-8 |dv|
  dq    scale sum ((r + fp) |dS| + P e) |k|, dk the same with |q| + 2^-8 of each,
        e = 2^-24 (dh + 2) (|do| |v| + |do| |out|) the error of dP - D
with r = 2^-8 or 0.  A probability below 2^-126 may become 0: of at most 2^12 terms each, with factors |dP - D| |q| up to 2^19
(2 * 128 * 4.5^2 and 16 * 4.5), that is 2^-95 more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import packed as opk          # noqa: E402
from paper_2410_07192_amd import synth    # noqa: E402

U32, U16, FLUSHED = 2.0 ** -24, 2.0 ** -8, 2.0 ** -95


def _mods():
    from paper_2410_07192_amd import binding as pf
    from paper_2410_07192_amd import device as dev
    return pf, dev


class Case:
    """Operands of one call: fused rows [Q | K | V | gap], NaN in rows of no sequence, on the device at `shift` elements."""

    def __init__(self, dtype, lens, h, kv, dh, causal, first=0, tail=0, gap=0, shift=0, seed=0, edit=None):
        pf, dev = _mods()
        self.dtype, self.h, self.kv, self.dh, self.causal = dtype, h, kv, dh, causal
        self.start = np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)
        self.T = T = int(self.start[-1]) + tail
        self.ld, self.ldo = (h + 2 * kv) * dh + gap, h * dh + gap
        rng = np.random.default_rng(seed)
        rnd = lambda *s: (synth.round_to_bf16(rng.standard_normal(s)) if dtype == "bf16" else rng.standard_normal(s).astype(np.float32))
        self.q, self.k, self.v, self.do = rnd(T, h, dh), rnd(T, kv, dh), rnd(T, kv, dh), rnd(T, h, dh)
        self.live = np.zeros(T, bool)
        self.live[first:self.start[-1]] = True
        if edit:
            edit(self)
            if dtype == "bf16":      # what the device gets: the checker has to start from the same numbers
                self.q, self.k, self.v, self.do = (torch.from_numpy(x).to(torch.bfloat16).float().numpy() for x in (self.q, self.k, self.v, self.do))
        for x in (self.q, self.k, self.v, self.do):
            x[~self.live] = np.nan
        self.shift = shift
        rows = np.full((T, self.ld), np.nan, np.float32)
        rows[:, :(h + 2 * kv) * dh] = np.concatenate([x.reshape(T, -1) for x in (self.q, self.k, self.v)], 1)
        self.qkv = self.put(rows)
        self.d_start = torch.from_numpy(self.start).cuda()
        self.desc = pf.packed_attn(pf.PF_DTYPE_BF16 if dtype == "bf16" else pf.PF_DTYPE_F32, T, len(lens), h, kv, dh, causal, self.ld, self.ld,
                                   self.ld, self.ldo)

    def put(self, a):
        t = torch.zeros(a.size + 64, dtype=torch.bfloat16 if self.dtype == "bf16" else torch.float32, device="cuda")
        t[self.shift:self.shift + a.size] = torch.from_numpy(np.ascontiguousarray(a, np.float32).reshape(-1)).cuda().to(t.dtype)
        return t

    def rows(self, t, ld):
        return t[self.shift:self.shift + self.T * ld].float().cpu().numpy().reshape(self.T, ld)

    def at(self, t, col=0):
        return t.data_ptr() + (self.shift + col) * t.element_size()

    def parts(self, t):
        return [self.at(t, c * self.dh) for c in (0, self.h, self.h + self.kv)]

    def forward(self, stream=None):
        pf, _ = _mods()
        out = self.put(np.full((self.T, self.ldo), 7.0))
        lse = torch.full((self.h, self.T), 7.0, device="cuda")
        pf.pf_op_attention_packed(self.desc, self.d_start.data_ptr(), *self.parts(self.qkv), self.at(out), lse.data_ptr(), stream)
        torch.cuda.synchronize()
        o = self.rows(out, self.ldo)
        assert (o[~self.live] == 7.0).all() and (o[:, self.h * self.dh:] == 7.0).all() and (lse.cpu().numpy()[:, ~self.live] == 7.0).all()
        return o[:, :self.h * self.dh].reshape(self.T, self.h, self.dh), lse.cpu().numpy()

    def backward(self, out, lse, stream=None):
        pf, _ = _mods()
        wide = lambda x: np.concatenate([x.reshape(self.T, -1), np.full((self.T, self.ldo - self.h * self.dh), np.nan)], 1)
        d_out, d_do, d_lse = self.put(wide(out)), self.put(wide(self.do)), torch.from_numpy(lse.astype(np.float32)).cuda()
        g = self.put(np.full((self.T, self.ld), 7.0))
        n = pf.pf_op_attention_packed_bwd_workspace(self.desc)
        ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
        pf.pf_op_attention_packed_bwd(self.desc, self.d_start.data_ptr(), *self.parts(self.qkv), self.at(d_out), self.at(d_do), d_lse.data_ptr(),
                                      *self.parts(g), ws.data_ptr(), n, stream)
        torch.cuda.synchronize()
        a = self.rows(g, self.ld)
        assert (a[~self.live] == 7.0).all() and (a[:, (self.h + 2 * self.kv) * self.dh:] == 7.0).all()
        cut = np.cumsum([self.h * self.dh, self.kv * self.dh, self.kv * self.dh])
        return (a[:, :cut[0]].reshape(self.T, self.h, self.dh), a[:, cut[0]:cut[1]].reshape(self.T, self.kv, self.dh),
                a[:, cut[1]:cut[2]].reshape(self.T, self.kv, self.dh))

    # ---- the checker and the tolerances
    def wide(self):
        clean = lambda x: np.where(self.live[:, None, None], x, 0).astype(np.float64)
        return [clean(x) for x in (self.q, self.k, self.v, self.do)]

    def rounding(self):
        stored = U16 if self.dtype == "bf16" else U32
        return stored, (U16 if self.dtype == "bf16" and self.dh in (64, 128) else 0.0)

    def check_forward(self, got=None, rows=None):
        """rows: the ones that are compared (default: all that are in a sequence)."""
        rows = self.live if rows is None else rows & self.live
        q, k, v, _ = self.wide()
        out, lse = opk.attention(q, k, v, self.start, self.causal)
        o, L = got or self.forward()
        stored, r = self.rounding()
        top, g = 0.0, self.h // self.kv
        for a, b in opk.spans(self.start):
            n = b - a
            for i in range(self.h):
                ka, va = k[a:b, i // g], np.abs(v[a:b, i // g])
                top = (np.abs(q[a:b, i]) @ np.abs(ka).T).max() / np.sqrt(self.dh)
                fp = U32 * ((self.dh + 4) * top + n + 16)
                p = np.exp(opk.scores(q[a:b, i], ka, self.causal) - lse[i, a:b, None])
                tol = (r + 2 * fp) * (p @ va) + stored * np.abs(out[a:b, i]) + FLUSHED
                r_ = rows[a:b]
                err = np.abs(o[a:b, i] - out[a:b, i])[r_]
                assert (err <= tol[r_]).all(), (a, b, i, (err / tol[r_]).max())
                assert (np.abs(L[i, a:b] - lse[i, a:b]) <= fp + 4 * U32 * np.abs(lse[i, a:b]))[r_].all(), (a, b, i)
        return o, L

    def saved(self):
        q, k, v, _ = self.wide()
        out, lse = opk.attention(q, k, v, self.start, self.causal)
        out = out.astype(np.float32)
        return (synth.round_to_bf16(out) if self.dtype == "bf16" else out).reshape(out.shape), lse.astype(np.float32)

    def check_backward(self, got=None, rows=None):
        rows = self.live if rows is None else rows & self.live
        q, k, v, do = self.wide()
        out, lse = self.saved()
        got = got or self.backward(out, lse)
        out, lse = out.astype(np.float64), lse.astype(np.float64)
        want = opk.attention_backward(q, k, v, out, do, lse, self.start, self.causal)
        stored, r = self.rounding()
        g, scale = self.h // self.kv, 1 / np.sqrt(self.dh)
        tol = [stored * np.abs(w) + FLUSHED for w in want]
        for a, b in opk.spans(self.start):
            n = b - a
            for i in range(self.h):
                j = i // g
                qi, ki, vi, di, oi = q[a:b, i], k[a:b, j], v[a:b, j], do[a:b, i], out[a:b, i]
                top = (np.abs(qi) @ np.abs(ki).T).max() * scale
                fp = U32 * ((self.dh + 4) * top + n * g + 16 + 4 * np.abs(lse[i, a:b]).max())
                p = np.exp(opk.scores(qi, ki, self.causal) - lse[i, a:b, None])
                ds = np.abs(p * (di @ vi.T - (di * oi).sum(-1, keepdims=True)))
                e = U32 * (self.dh + 2) * (np.abs(di) @ np.abs(vi).T + (np.abs(di) * np.abs(oi)).sum(-1, keepdims=True))
                w = (r + fp) * ds + p * e
                tol[0][a:b, i] += scale * (w @ np.abs(ki))
                tol[1][a:b, j] += scale * (w.T @ np.abs(qi))
                tol[2][a:b, j] += (r + fp) * (p.T @ np.abs(di))
        for name, x, w, t in zip(("dq", "dk", "dv"), got, want, tol):
            bad = ~(np.abs(x - w)[rows] <= t[rows])
            assert not bad.any(), (name, int(bad.sum()), np.abs((x - w)[rows] / np.maximum(t[rows], 1e-30)).max())
        return got


# (dtype, lengths, heads, K/V heads, d_head, rows before, rows behind)
SHAPES = [
    ("bf16", [1], 1, 1, 64, 0, 0),                                 # one token in all
    ("bf16", [1], 8, 1, 128, 3, 2),
    ("f32", [1, 1, 1, 2], 2, 1, 64, 0, 0),
    ("f32", [0, 5, 0, 0, 33, 1, 0], 4, 2, 32, 2, 40),              # empty sequences, rows in none
    ("f32", [32, 64, 31], 3, 1, 128, 0, 1),
    ("f32", [40, 9], 3, 3, 8, 1, 0),
    ("f32", [70, 3, 100], 2, 2, 16, 0, 5),
    ("bf16", [17, 60], 4, 4, 16, 0, 3),
    ("bf16", [100, 7], 6, 2, 32, 0, 0),
    ("bf16", [3] * 90, 4, 2, 64, 0, 0),                            # more sequences than a wave has lanes
    ("bf16", [0] * 70 + [50] + [0] * 70 + [9, 200], 4, 1, 64, 7, 9),
    ("bf16", [64, 128, 64], 8, 8, 64, 0, 0),                       # whole tiles
    ("bf16", [63, 65, 127, 129, 1], 12, 12, 64, 0, 64),
    ("bf16", [333], 16, 2, 128, 0, 0),
    ("bf16", [257, 30, 511], 8, 2, 128, 5, 17),
    ("bf16", [257, 30, 511], 5, 5, 128, 0, 0),
    ("bf16", [700, 1, 90], 7, 1, 64, 0, 0),                        # a group that is no power of two
    ("bf16", [1200, 40], 12, 2, 128, 0, 0),
    ("bf16", [900, 900], 32, 4, 64, 0, 300),
    ("f32", [300, 77], 6, 3, 64, 0, 0),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,lens,h,kv,dh,first,tail", SHAPES, ids=lambda x: "x".join(map(str, x[:4])) if isinstance(x, list) else str(x))
def test_forward_and_backward(dtype, lens, h, kv, dh, first, tail, causal):
    c = Case(dtype, lens, h, kv, dh, causal, first, tail, seed=len(lens) + h)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype,dh,gap,shift", [("bf16", 64, 8, 8), ("bf16", 128, 24, 0), ("bf16", 64, 1, 0), ("bf16", 64, 8, 3), ("bf16", 128, 4, 4),
                                                ("f32", 64, 8, 4), ("f32", 32, 3, 0), ("f32", 128, 0, 1)])
def test_strides_and_alignment(dtype, dh, gap, shift):
    c = Case(dtype, [90, 1, 140], 4, 2, dh, True, 2, 3, gap=gap, shift=shift, seed=gap + shift)
    c.check_forward()
    c.check_backward()


def test_one_sequence_without_boundaries():
    pf, _ = _mods()
    c = Case("bf16", [150], 4, 2, 64, True, seed=5)
    want, want_g = c.forward(), None
    saved = c.saved()
    want_g = c.backward(*saved)
    c.desc.n_seq = 0
    c.d_start = torch.empty(0, dtype=torch.int32, device="cuda")
    assert c.d_start.data_ptr() == 0
    got = c.forward()
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    assert all(np.array_equal(a, b) for a, b in zip(c.backward(*saved), want_g))


@pytest.mark.parametrize("dtype,h,kv,dh", [("bf16", 4, 2, 64), ("bf16", 8, 1, 128), ("bf16", 2, 2, 32), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_values_that_a_row_does_not_see_do_not_reach_it(dtype, h, kv, dh, causal):
    """Infinities and NaN in one sequence (and, causal, in the last rows of another) leave the rest as it would be without them."""
    lens = [70, 45, 20, 130, 9]

    def poison(c):
        a, b = c.start[1:3]
        for x in (c.q, c.k, c.v, c.do):
            x[a:b:3] = np.nan
            x[a + 1:b:3] = np.inf
        if causal:
            for x in (c.k, c.v):
                x[c.start[4] - 6:c.start[4]] = -np.inf
            x = c.v
            x[c.start[4] - 3] = np.nan

    good, bad = Case(dtype, lens, h, kv, dh, causal, 1, 2, seed=3), Case(dtype, lens, h, kv, dh, causal, 1, 2, seed=3, edit=poison)
    clean = np.ones(good.T, bool)
    clean[good.start[1]:good.start[2]] = False
    late = clean.copy()
    if causal:
        late[good.start[4] - 6:good.start[4]] = False
    o, _ = good.check_forward(bad.forward(), late)      # the checker's values without them, to the same tolerance
    assert np.isnan(o[good.start[1]:good.start[2]]).any()
    out, lse = good.saved()

    def poison_qd(c):   # the backward pass: other sequences' rows, and rows of this one that come before (causal queries)
        poison_all = slice(c.start[1], c.start[2])
        for x in (c.q, c.k, c.v, c.do):
            x[poison_all][::2] = np.nan
            x[poison_all][1::2] = np.inf
        if causal:
            for x in (c.q, c.do):
                x[c.start[3]:c.start[3] + 5] = np.nan

    bad = Case(dtype, lens, h, kv, dh, causal, 1, 2, seed=3, edit=poison_qd)
    keys = clean.copy()
    if causal:
        keys[good.start[3]:good.start[3] + 5] = False
    good.check_backward(bad.backward(out, lse), keys)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_large_scores(dtype, dh):
    """Scores of a few hundred: the maximum moves from tile to tile."""
    def big(c):
        c.q *= 16
        ramp = (1 + np.arange(c.T) % 7)[:, None, None].astype(np.float32)
        c.k *= ramp
    c = Case(dtype, [300, 77], 4, 2, dh, True, seed=9, edit=big)
    c.check_forward()
    c.check_backward()


def test_lowest_and_infinite_scores():
    """Keys whose scores are the type's lowest value or -inf get probability 0; a row that sees only -inf has no softmax."""
    def edit(c):
        c.q[:] = 0
        c.q[:, :, 0] = 1
        c.k[:, :, 0] = 0
        c.k[10:20, :, 0] = -3e38
        c.k[30:40, :, 0] = -np.inf
        c.k[c.start[1]:, :, 0] = -np.inf
    for dtype, dh in (("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 32)):
        c = Case(dtype, [100, 30], 2, 1, dh, True, seed=2, edit=edit)
        o, lse = c.forward()
        a = np.arange(100)
        seen = [v for v in range(100) if not (10 <= v < 20 or 30 <= v < 40)]
        s = np.where(np.isin(a, seen), 0.0, -np.inf)
        for row in (9, 25, 45, 99):
            p = np.exp(s[:row + 1])
            want = (p[:, None] * c.v[:row + 1, 0]).sum(0) / p.sum()
            tol = (2 * U16 + 1e-5) * (p[:, None] * np.abs(c.v[:row + 1, 0])).sum(0) / p.sum()
            assert (np.abs(o[row, 0] - want) <= tol).all()
            assert abs(lse[0, row] - np.log(p.sum())) < 1e-5
        assert np.isnan(o[100:]).all()


def test_the_same_results_every_time_and_on_another_stream():
    c = Case("bf16", [400, 33, 270], 8, 2, 64, True, seed=4)
    saved = c.saved()
    first = c.forward() + c.backward(*saved)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for s in (None, st.cuda_stream):
        torch.cuda.synchronize()
        again = c.forward(s) + c.backward(*saved, s)
        assert all(np.array_equal(a, b) for a, b in zip(first, again))


def test_captured_with_other_lengths():
    """A graph captured once is replayed with other boundaries in the same buffers."""
    pf, _ = _mods()
    c = Case("bf16", [200, 100], 4, 2, 64, True, seed=6)
    out, lse = c.put(np.zeros((c.T, c.ldo))), torch.zeros(c.h, c.T, device="cuda")
    g = c.put(np.zeros((c.T, c.ld)))
    do = c.put(c.do.reshape(c.T, -1))
    n = pf.pf_op_attention_packed_bwd_workspace(c.desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call(stream):
        pf.pf_op_attention_packed(c.desc, c.d_start.data_ptr(), *c.parts(c.qkv), c.at(out), lse.data_ptr(), stream)
        pf.pf_op_attention_packed_bwd(c.desc, c.d_start.data_ptr(), *c.parts(c.qkv), c.at(out), c.at(do), lse.data_ptr(), *c.parts(g), ws.data_ptr(), n,
                                      stream)
    call(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream().cuda_stream)
    for start in ([0, 200, 300], [0, 7, 300], [5, 290, 300], [0, 0, 300], [0, 150, 180]):
        c.d_start.copy_(torch.tensor(start, dtype=torch.int32))
        for x in (out, lse, g):
            x.zero_()
        call(torch.cuda.current_stream().cuda_stream)
        want = [x.clone() for x in (out, lse, g)]
        for x in (out, lse, g):
            x.zero_()
        ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, g), want)), start


def test_far_rows():
    """Rows whose offsets pass 32 bits (a wide stride): only the last sequence is looked at."""
    pf, _ = _mods()
    h, kv, dh, n, ld = 2, 1, 64, 40, 1 << 20
    T = (1 << 12) + 200
    rows = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")       # 9 GB: most of it is never touched
    gen = torch.Generator(device="cuda").manual_seed(0)
    last = torch.randn(n, (h + 2 * kv) * dh, device="cuda", generator=gen).to(torch.bfloat16)
    view = rows.view(T, ld)
    view[T - n:, :last.shape[1]] = last
    start = torch.tensor([T - n, T], dtype=torch.int32, device="cuda")
    small = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    res = []
    for t, s, base, stride in ((T, start, rows, ld), (n, small, last, last.shape[1])):
        desc = pf.packed_attn(pf.PF_DTYPE_BF16, t, 1, h, kv, dh, True, stride, stride, stride)
        out, lse = torch.zeros(t, h * dh, dtype=torch.bfloat16, device="cuda"), torch.zeros(h, t, device="cuda")
        g = torch.zeros_like(base)
        p = lambda x: [x.data_ptr() + 2 * dh * c for c in (0, h, h + kv)]
        pf.pf_op_attention_packed(desc, s.data_ptr(), *p(base), out.data_ptr(), lse.data_ptr())
        m = pf.pf_op_attention_packed_bwd_workspace(desc)
        ws = torch.empty(m, dtype=torch.uint8, device="cuda")
        pf.pf_op_attention_packed_bwd(desc, s.data_ptr(), *p(base), out.data_ptr(), out.data_ptr(), lse.data_ptr(), *p(g), ws.data_ptr(), m)
        torch.cuda.synchronize()
        res.append((out[t - n:].clone(), g.view(t, stride)[t - n:, :last.shape[1]].clone()))
    # blocks of rows begin elsewhere, so sums come in another order: half a bf16 step of rounding each side, of values up to the largest
    for a, b in zip(*res):
        assert float((a.float() - b.float()).abs().max()) <= 4 * U16 * float(b.float().abs().max())
