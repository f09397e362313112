"""The operators on packed sequences as a user calls them: batches whose sequences have different lengths and lie one behind the
other in [tokens][...] buffers, sequence s in rows seq_start[s] .. seq_start[s + 1] - 1.

Four kinds of case:
  attn       softmax(Q K^T / sqrt(d_head)) V within each sequence, grouped heads; result: output and log-sum-exp
  attn_bwd   its gradients from the saved output and log-sum-exp; result: dQ, dK, dV
  embed      scaled token rows plus the row of the position within the sequence; result: hidden states
  embed_bwd  its gradients; result: the two tables' gradients in fp32
"""
import math
import random

import numpy as np
import torch

own = False


def _attn(name, kind, dtype, causal, heads, kv, dh, n_seq, longest, tail=0):
    c = dict(kind=kind, dtype=dtype, causal=causal, heads=heads, kv=kv, dh=dh, n_seq=n_seq, longest=longest, tail=tail)
    return dict(name=name, **c) if name else c


def _embed(name, kind, dtype, d, vocab, n_seq, longest, tail=0):
    c = dict(kind=kind, dtype=dtype, d=d, vocab=vocab, n_seq=n_seq, longest=longest, tail=tail)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the fp32 encoder layer of cfg1 on four sequences of different lengths
        _attn("attn_fp32", "attn", "f32", False, 4, 4, 64, 4, 128),
        # one prompt of odd length before its first token is generated: latency counts
        _attn("attn_prompt", "attn", "bf16", True, 16, 2, 128, 1, 333),
        # cfg2's encoder heads on a batch of documents up to 512 tokens, in a buffer with room behind the last one
        _attn("attn_encoder", "attn", "bf16", False, 12, 12, 64, 32, 512, tail=200),
        # prompts of very different lengths with cfg3's query heads and few K/V heads
        _attn("attn_prefill", "attn", "bf16", True, 16, 2, 128, 16, 2048),
        # two long documents at once
        _attn("attn_long", "attn", "bf16", True, 32, 4, 128, 2, 8192),
        # gradients of the fp32 layer
        _attn("attn_bwd_fp32", "attn_bwd", "f32", True, 4, 2, 64, 4, 128),
        # a training microbatch of cfg4's size (d_head 64), packed, with grouped heads
        _attn("attn_bwd_batch", "attn_bwd", "bf16", True, 16, 4, 64, 12, 1024, tail=77),
        # training on long documents with d_head 128
        _attn("attn_bwd_long", "attn_bwd", "bf16", True, 16, 2, 128, 3, 4096),
        # one request to the encoder of cfg2
        _embed("embed_request", "embed", "bf16", 768, 30522, 1, 128),
        # a packed batch for cfg3's decoder
        _embed("embed_batch", "embed", "bf16", 2048, 50257, 40, 1024, tail=111),
        # a small fp32 model's step
        _embed("embed_bwd_small", "embed_bwd", "f32", 512, 10007, 5, 200),
        # a training microbatch of cfg4's size
        _embed("embed_bwd_batch", "embed_bwd", "bf16", 1024, 50257, 16, 1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: sizes log-uniform, head counts, d_head and lengths as they come, no costlier than the
    largest listed case of its kind."""
    cost = lambda c: max(work(c)["flops"] / (2 if c["dtype"] == "f32" else 50), work(c)["bytes"])
    most = {}
    for c in listed():
        key = c["kind"] + (c["dtype"] if c["kind"].startswith("attn") else "")
        most[key] = max(most.get(key, 0.0), cost(c))
    while True:
        kind = rng.choice(["attn", "attn", "attn_bwd", "attn_bwd", "embed", "embed_bwd"])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        tail = rng.choice([0, 0, rng.randint(1, 300)])
        if kind.startswith("attn"):
            small = dtype == "f32"
            kv = _log(rng, 1, 4 if small else 16)
            heads = kv * rng.choice([1, 1, 2, 3, 4, 5, 8])
            longest = _log(rng, 1, 256) if small else _log(rng, 16, 8192 if kind == "attn" else 4096)
            c = _attn(None, kind, dtype, rng.random() < 0.7, heads, kv, rng.choice([32, 64] if small else [64, 128]),
                      _log(rng, 1, 8 if small else 128), longest, tail)
            ok = heads <= (8 if small else 32) and c["n_seq"] * heads * longest ** 2 <= 1 << 32
        else:
            c = _embed(None, kind, dtype, 8 * _log(rng, 32, 256), _log(rng, 500, 50257), _log(rng, 1, 200), _log(rng, 1, 2048),
                       tail)
            ok = True
        if ok and cost(c) <= most[kind + (dtype if kind.startswith("attn") else "")]:
            return c


def _lengths(c):
    """Lengths of the sequences: the longest one is there, the others spread over the logarithm from a sixteenth of it."""
    r = random.Random(c["n_seq"] * 1000003 + c["longest"])
    return [c["longest"]] + [max(1, _log(r, max(1.0, c["longest"] / 16), c["longest"])) for _ in range(c["n_seq"] - 1)]


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    lens = _lengths(c)
    random.Random(seed).shuffle(lens)
    start = torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
    tokens = sum(lens) + c["tail"]
    dt = _type(c)
    s = {"case": c, "start": start, "tokens": tokens, "kept": {}}
    if c["kind"].startswith("attn"):
        h, kv, dh = c["heads"], c["kv"], c["dh"]
        # the fused projection's output: Q heads | K heads | V heads in every row
        s["qkv"] = normal(tokens, (h + 2 * kv) * dh).to(dt)
        s["out"] = torch.zeros(tokens, h * dh, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(h, tokens, device="cuda")
        if c["kind"] == "attn_bwd":
            got = _plain_attn(s)
            s["out"], s["lse"] = got["out"], got["lse"]
            s["dout"] = normal(tokens, h * dh).to(dt)
            s["dqkv"] = torch.zeros_like(s["qkv"])
    else:
        d, vocab = c["d"], c["vocab"]
        # a token's frequency falls with its id, as in vocabularies ordered by frequency: p(id) = log((id + 2) / (id + 1)) / log(V + 1)
        u = torch.rand(tokens, device="cuda", generator=gen, dtype=torch.float64)
        s["ids"] = (torch.exp(u * math.log(vocab + 1)).floor().to(torch.int64) - 1).clamp(0, vocab - 1).to(torch.int32)
        s["scale"] = math.sqrt(d)
        if c["kind"] == "embed":
            s["tok"], s["pos"] = (normal(vocab, d) * 0.02).to(dt), (normal(c["longest"], d) * 0.02).to(dt)
            s["x"] = torch.zeros(tokens, d, dtype=dt, device="cuda")
        else:
            s["dx"] = (normal(tokens, d) * 1e-3).to(dt)
            s["dtok"] = torch.zeros(vocab, d, device="cuda")
            s["dpos"] = torch.zeros(c["longest"], d, device="cuda")
    return s


# ---- the operators in elementary operations --------------------------------------------------------------------------------
def _padded(s):
    """Row of every place of the batch padded to [sequences][longest], whether it is one, and where results go (one row more
    than there is takes those of places that are none)."""
    start = s["start"].long()
    row = start[:-1, None] + torch.arange(s["case"]["longest"], device=start.device)
    valid = row < start[1:, None]
    return row.clamp(max=s["tokens"] - 1), valid, torch.where(valid, row, s["tokens"])


def _heads_of(s, row):
    """Q [n][kv][group * L][dh], K and V [n][kv][L][dh] in fp32."""
    c = s["case"]
    n, L = row.shape
    h, kv, dh = c["heads"], c["kv"], c["dh"]
    x = s["qkv"].float()[row].view(n, L, h + 2 * kv, dh)
    q = x[:, :, :h].view(n, L, kv, h // kv, dh).permute(0, 2, 3, 1, 4).reshape(n, kv, h // kv * L, dh)
    k, v = (x[:, :, a:a + kv].permute(0, 2, 1, 3).contiguous() for a in (h, h + kv))
    return q, k, v


def _by_query(s, x, row):
    """[tokens][heads * dh] -> [n][kv][group * L][dh] in fp32."""
    c = s["case"]
    n, L = row.shape
    g = c["heads"] // c["kv"]
    return x.float()[row].view(n, L, c["kv"], g, c["dh"]).permute(0, 2, 3, 1, 4).reshape(n, c["kv"], g * L, c["dh"])


def _to_rows(s, x, to, group):
    """[n][kv][group * L][dh] -> [tokens][kv * group * dh]."""
    c = s["case"]
    n, L = to.shape
    y = x.view(n, c["kv"], group, L, c["dh"]).permute(0, 3, 1, 2, 4).reshape(n, L, -1)
    out = torch.zeros(s["tokens"] + 1, y.shape[-1], device=y.device)
    out[to] = y
    return out[:-1].to(_type(c))


def _visible(s, valid):
    L = valid.shape[1]
    m = valid[:, None, None, None, :]
    if s["case"]["causal"]:
        at = torch.arange(L, device=valid.device)
        m = m & (at[None, :] <= at[:, None])
    return m                                                      # [n][1][1][1 or L][L]


def _plain_attn(s):
    c = s["case"]
    row, valid, to = _padded(s)
    n, L = row.shape
    h, kv, dh = c["heads"], c["kv"], c["dh"]
    q, k, v = _heads_of(s, row)
    sc = torch.matmul(q * (1.0 / math.sqrt(dh)), k.transpose(-1, -2).contiguous()).view(n, kv, h // kv, L, L)
    sc.masked_fill_(~_visible(s, valid), -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, kv, -1, L), v) / total.view(n, kv, -1, 1)
    lse = torch.zeros(h, s["tokens"] + 1, device="cuda")
    lse[:, to] = (top + total.log()).view(n, h, L).permute(1, 0, 2)
    return {"out": _to_rows(s, o, to, h // kv), "lse": lse[:, :-1].contiguous()}


def _plain_attn_bwd(s):
    c = s["case"]
    row, valid, to = _padded(s)
    n, L = row.shape
    h, kv, dh = c["heads"], c["kv"], c["dh"]
    scale = 1.0 / math.sqrt(dh)
    q, k, v = _heads_of(s, row)
    o, do = _by_query(s, s["out"], row), _by_query(s, s["dout"], row)
    real = valid[:, None, None, :, None].expand(n, kv, h // kv, L, 1).reshape(n, kv, -1, 1)
    do = do * real
    lse = s["lse"][:, row].view(kv, h // kv, n, L).permute(2, 0, 1, 3)
    p = torch.matmul(q * scale, k.transpose(-1, -2).contiguous()).view(n, kv, h // kv, L, L)
    p.sub_(lse[..., None])
    p.masked_fill_(~(_visible(s, valid) & valid[:, None, None, :, None]), -math.inf)
    p = p.exp_().view(n, kv, -1, L)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    dk = torch.matmul(ds.transpose(-1, -2), q) * scale
    dq = torch.matmul(ds, k) * scale
    return {"dq": _to_rows(s, dq, to, h // kv), "dk": _to_rows(s, dk, to, 1), "dv": _to_rows(s, dv, to, 1)}


def _places(s):
    """Position of every row within its sequence, and whether it is in one."""
    start = s["start"].long()
    t = torch.arange(s["tokens"], device=start.device)
    nth = (start[None, :] <= t[:, None]).sum(1) - 1
    return t - start[nth], nth < s["case"]["n_seq"]


def _plain_embed(s):
    place, real = _places(s)
    place = torch.where(real, place, 0)
    x = s["tok"][s["ids"].long()].float() * s["scale"] + s["pos"][place].float()
    return (x * real[:, None]).to(_type(s["case"]))


def _plain_embed_bwd(s):
    place, real = _places(s)
    place = torch.where(real, place, 0)
    dx = s["dx"].float() * real[:, None]
    dtok, dpos = torch.zeros_like(s["dtok"]), torch.zeros_like(s["dpos"])
    dtok.index_add_(0, s["ids"].long(), dx)
    dpos.index_add_(0, place, dx)
    return {"dtok": dtok * s["scale"], "dpos": dpos}


# ---- the calls of the framework -----------------------------------------------------------------------------------------------
def _own(s):
    from paper_2410_07192_amd import binding as pf
    c, kept = s["case"], s["kept"]
    stream = torch.cuda.current_stream().cuda_stream
    dt = pf.PF_DTYPE_BF16 if c["dtype"] == "bf16" else pf.PF_DTYPE_F32
    start = s["start"].data_ptr()
    if c["kind"].startswith("attn"):
        h, kv, dh = c["heads"], c["kv"], c["dh"]
        ld = (h + 2 * kv) * dh
        parts = lambda x: [x.data_ptr() + at * dh * x.element_size() for at in (0, h, h + kv)]
        if "desc" not in kept:
            kept["desc"] = pf.packed_attn(dt, s["tokens"], c["n_seq"], h, kv, dh, c["causal"], ld_q=ld, ld_k=ld, ld_v=ld)
            if c["kind"] == "attn_bwd":
                n = pf.pf_op_attention_packed_bwd_workspace(kept["desc"])
                kept["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        if c["kind"] == "attn":
            pf.pf_op_attention_packed(kept["desc"], start, *parts(s["qkv"]), s["out"].data_ptr(), lse=s["lse"].data_ptr(),
                                      stream=stream)
            return {"out": s["out"], "lse": s["lse"]}
        pf.pf_op_attention_packed_bwd(kept["desc"], start, *parts(s["qkv"]), s["out"].data_ptr(), s["dout"].data_ptr(),
                                      s["lse"].data_ptr(), *parts(s["dqkv"]), kept["ws"].data_ptr(), kept["ws"].numel(),
                                      stream=stream)
        g = s["dqkv"]
        return {"dq": g[:, :h * dh], "dk": g[:, h * dh:(h + kv) * dh], "dv": g[:, (h + kv) * dh:]}
    if c["kind"] == "embed":
        pf.pf_op_embed_packed(dt, s["ids"].data_ptr(), s["tok"].data_ptr(), s["pos"].data_ptr(), start, c["n_seq"], s["scale"],
                              s["x"].data_ptr(), s["tokens"], c["longest"], c["d"], c["vocab"], stream=stream)
        return s["x"]
    if "ws" not in kept:
        n = pf.pf_op_embed_packed_bwd_workspace(s["tokens"], c["longest"], c["d"], c["vocab"])
        kept["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    pf.pf_op_embed_packed_bwd(dt, s["dx"].data_ptr(), s["ids"].data_ptr(), start, c["n_seq"], s["scale"], s["dtok"].data_ptr(),
                              s["dpos"].data_ptr(), 0, kept["ws"].data_ptr(), kept["ws"].numel(), s["tokens"], c["longest"],
                              c["d"], c["vocab"], stream=stream)
    return {"dtok": s["dtok"], "dpos": s["dpos"]}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"attn": _plain_attn, "attn_bwd": _plain_attn_bwd, "embed": _plain_embed, "embed_bwd": _plain_embed_bwd}[kind](state)


# ---- what a pass cannot do without, and its results in 64 bits -----------------------------------------------------------------
def work(case):
    c, lens = case, _lengths(case)
    size, T = (2 if c["dtype"] == "bf16" else 4), sum(lens)
    if c["kind"].startswith("attn"):
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens) * c["heads"]
        q, kv, lse = T * c["heads"] * c["dh"] * size, T * c["kv"] * c["dh"] * size, T * c["heads"] * 4
        if c["kind"] == "attn":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * c["dh"] * pairs}
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * c["dh"] * pairs}
    d, V = c["d"], c["vocab"]
    if c["kind"] == "embed_bwd":
        return {"bytes": T * (d * size + 4) + (V + c["longest"]) * d * 4, "flops": 2 * T * d}
    ids = np.arange(V)
    p = np.log((ids + 2) / (ids + 1)) / math.log(V + 1)
    touched = float(np.sum(1.0 - (1.0 - p) ** T))                 # expected number of different ids
    return {"bytes": T * (d * size + 4) + (touched + c["longest"]) * d * size, "flops": 2 * T * d}


def exact(case, seed):
    s = prepare(case, seed)
    c, T = case, s["tokens"]
    edges = s["start"].tolist()
    spans = list(zip(edges[:-1], edges[1:]))
    f64 = dict(dtype=torch.float64, device="cuda")
    if not c["kind"].startswith("attn"):
        ids = s["ids"].long()
        if c["kind"] == "embed":
            x = torch.zeros(T, c["d"], **f64)
            for a, b in spans:
                x[a:b] = s["tok"][ids[a:b]].double() * s["scale"] + s["pos"][:b - a].double()
            return x
        dtok, dpos = torch.zeros(c["vocab"], c["d"], **f64), torch.zeros(c["longest"], c["d"], **f64)
        for a, b in spans:
            dx = s["dx"][a:b].double()
            dtok.index_add_(0, ids[a:b], dx * s["scale"])
            dpos[:b - a] += dx
        return {"dtok": dtok, "dpos": dpos}
    h, kv, dh = c["heads"], c["kv"], c["dh"]
    x = s["qkv"].view(T, h + 2 * kv, dh)
    out, lse = torch.zeros(T, h, dh, **f64), torch.zeros(h, T, **f64)
    dq, dk, dv = torch.zeros(T, h, dh, **f64), torch.zeros(T, kv, dh, **f64), torch.zeros(T, kv, dh, **f64)
    for a, b in spans:
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1) if c["causal"] else None
        for i in range(h):
            j = h + i // (h // kv)
            q, k, v = x[a:b, i].double(), x[a:b, j].double(), x[a:b, j + kv].double()
            sc = q @ k.t().contiguous() / math.sqrt(dh)
            if hidden is not None:
                sc = sc.masked_fill(hidden, -math.inf)
            if c["kind"] == "attn":
                lse[i, a:b] = torch.logsumexp(sc, -1)
                out[a:b, i] = torch.exp(sc - lse[i, a:b, None]) @ v
                continue
            p = torch.exp(sc - s["lse"][i, a:b, None].double())
            do, o = (s[n].view(T, h, dh)[a:b, i].double() for n in ("dout", "out"))
            ds = p * (do @ v.t().contiguous() - (do * o).sum(-1, keepdim=True)) / math.sqrt(dh)
            dq[a:b, i] = ds @ k
            dk[a:b, j - h] += ds.t() @ q
            dv[a:b, j - h] += p.t() @ do
    if c["kind"] == "attn":
        return {"out": out.view(T, -1), "lse": lse}
    return {"dq": dq.view(T, -1), "dk": dk.view(T, -1), "dv": dv.view(T, -1)}
