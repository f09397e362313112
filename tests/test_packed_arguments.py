"""What the operators on packed sequences refuse: decided on the host before anything is launched, so without a GPU."""
import ctypes as C

import pytest

from paper_2410_07192_amd import binding as pf

P = 1 << 20      # an aligned address nothing reads: every call here is refused


def _desc(**kw):
    a = dict(dtype=pf.PF_DTYPE_BF16, tokens=100, n_seq=3, n_heads=8, n_kv_heads=2, d_head=64, causal=True)
    a.update(kw)
    return pf.packed_attn(**a)


def _fwd(desc, start=P, q=P, k=P, v=P, out=P, lse=P):
    pf.pf_op_attention_packed(desc, start, q, k, v, out, lse)


def _bwd(desc, start=P, ptr=P, lse=P, ws=P, ws_bytes=1 << 40, **kw):
    p = dict.fromkeys(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), ptr)
    p.update(kw)
    pf.pf_op_attention_packed_bwd(desc, start, p["q"], p["k"], p["v"], p["out"], p["dout"], lse, p["dq"], p["dk"], p["dv"], ws,
                                  ws_bytes)


BAD_DESC = [dict(dtype=7), dict(tokens=0), dict(tokens=-5), dict(tokens=1 << 31), dict(tokens=1 << 25), dict(n_seq=-1), dict(n_seq=0),
            dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=6, n_kv_heads=4), dict(n_kv_heads=-2), dict(d_head=48), dict(d_head=256),
            dict(ld_q=8 * 64 - 1), dict(ld_k=2 * 64 - 8), dict(ld_v=-128), dict(ld_out=64)]


@pytest.mark.parametrize("kw", BAD_DESC, ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items()))
def test_attention_descriptions_refused(kw):
    for call in (_fwd, _bwd):
        with pytest.raises(pf.PipeFillError) as e:
            call(_desc(**kw))
        assert e.value.code == pf.PF_ERR_ARG and "pf_op_attention_packed" in e.value.msg


def test_attention_pointers_refused():
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(start=None), dict(q=P + 1), dict(out=P + 1), dict(lse=P + 2),
               dict(start=P + 2)):
        with pytest.raises(pf.PipeFillError) as e:
            _fwd(_desc(), **kw)
        assert e.value.code == pf.PF_ERR_ARG
    for kw in (dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(lse=None), dict(ws=None), dict(ws=P + 16), dict(dk=P + 1)):
        with pytest.raises(pf.PipeFillError) as e:
            _bwd(_desc(), **kw)
        assert e.value.code == pf.PF_ERR_ARG
    assert pf.lib.pf_op_attention_packed(None, P, P, P, P, P, None, None) == pf.PF_ERR_ARG
    assert pf.lib.pf_op_attention_packed_bwd_workspace(None) == pf.PF_ERR_ARG


def test_attention_workspace():
    n = pf.pf_op_attention_packed_bwd_workspace(_desc())
    assert n >= 8 * 100 * 4
    with pytest.raises(pf.PipeFillError) as e:
        _bwd(_desc(), ws_bytes=n - 1)
    assert e.value.code == pf.PF_ERR_NOMEM and str(n) in e.value.msg
    with pytest.raises(pf.PipeFillError):
        pf.pf_op_attention_packed_bwd_workspace(_desc(d_head=24))


def _embed(dtype=pf.PF_DTYPE_BF16, ids=P, tok=P, pos=P, start=P, n_seq=2, x=P, tokens=50, S=64, d=64, V=100):
    pf.pf_op_embed_packed(dtype, ids, tok, pos, start, n_seq, 1.0, x, tokens, S, d, V)


def _embed_bwd(dtype=pf.PF_DTYPE_BF16, ids=P, tok=P, pos=P, start=P, n_seq=2, x=P, tokens=50, S=64, d=64, V=100, ws=P, ws_bytes=1 << 40):
    pf.pf_op_embed_packed_bwd(dtype, x, ids, start, n_seq, 1.0, tok, pos, 0, ws, ws_bytes, tokens, S, d, V)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(ids=None), dict(tok=None), dict(x=None), dict(start=None), dict(n_seq=0), dict(n_seq=-1),
                                dict(tokens=0), dict(tokens=(1 << 26) + 1), dict(tokens=1 << 25, d=2048), dict(S=0), dict(d=0), dict(d=60),
                                dict(V=0), dict(V=(1 << 24) + 1), dict(S=(1 << 24) + 1), dict(tok=P + 8), dict(pos=P + 8), dict(x=P + 8),
                                dict(ids=P + 1)], ids=str)
def test_embedding_arguments_refused(kw):
    for call in (_embed, _embed_bwd):
        with pytest.raises(pf.PipeFillError) as e:
            call(**kw)
        assert e.value.code == pf.PF_ERR_ARG and "pf_op_embed_packed" in e.value.msg


def test_embedding_workspace():
    n = pf.pf_op_embed_packed_bwd_workspace(50, 64, 64, 100)
    with pytest.raises(pf.PipeFillError) as e:
        _embed_bwd(ws_bytes=n - 1)
    assert e.value.code == pf.PF_ERR_NOMEM
    for kw in (dict(ws=None), dict(ws=P + 64)):
        with pytest.raises(pf.PipeFillError) as e:
            _embed_bwd(**kw)
        assert e.value.code == pf.PF_ERR_ARG
    with pytest.raises(pf.PipeFillError):
        pf.pf_op_embed_packed_bwd_workspace(50, 64, 63, 100)


def test_struct_size_matches_the_header():
    assert C.sizeof(pf.pf_packed_attn) == 64


@pytest.mark.parametrize("kw", [dict(ld_q=(1 << 24) + 8), dict(ld_k=(1 << 24) + 8), dict(ld_v=1 << 40), dict(ld_out=(1 << 24) + 8),
                                dict(tokens=1 << 24, n_heads=16), dict(n_seq=1 << 31), dict(n_heads=1 << 27, n_kv_heads=1 << 27)], ids=str)
def test_attention_sizes_refused(kw):
    if kw.get("n_seq", 0) >= 1 << 31:
        desc = _desc()
        desc.n_seq = -(1 << 31)      # what a 32-bit field makes of it
    else:
        desc = _desc(**kw)
    for call in (_fwd, _bwd):
        with pytest.raises(pf.PipeFillError) as e:
            call(desc)
        assert e.value.code == pf.PF_ERR_ARG
