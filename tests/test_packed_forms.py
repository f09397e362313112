"""Which kernel a call of packed attention takes is decided on the host, by sizes and alignment: here without a GPU, so that a change of the rules
that leaves a form of the kernels without a GPU test fails."""
import ctypes as C
import random

import pytest

from paper_2410_07192_amd import binding as pf

FORMS = ("fp32 products", "S1", "S2", "W1", "W2", "W4")     # tiles shared by four waves, a block's keys in 1 or 2 parts; independent waves, 1, 2 or 4 to a block


def route(dtype, rows, n_seq, h, kv, dh, causal, misaligned=False, ld=0):
    """(form of the forward; "o", "k", "q": blocks of the forward, of dK/dV and of dQ taken longest first; heads of a workgroup; parts of dK/dV)"""
    f = pf.lib.pf_attention_packed_route
    f.restype, f.argtypes = C.c_int32, [C.POINTER(pf.pf_packed_attn), C.c_int32]
    desc = pf.packed_attn(pf.PF_DTYPE_F32 if dtype == "f32" else pf.PF_DTYPE_BF16, rows, n_seq, h, kv, dh, causal, ld, ld, ld, 0)
    r = f(C.byref(desc), int(misaligned))
    assert r >= 0
    return FORMS[r & 255], "".join(c for i, c in enumerate("okq") if r >> 8 + i & 1), r >> 12 & 15, r >> 16 & 255


def ragged(n, longest, seed):
    """Lengths spread over the logarithm from a sixteenth of the longest."""
    r = random.Random(seed)
    return [max(1, int(longest * 16 ** -r.random())) for _ in range(n)]


# Batches whose blocks are taken in order of length, in every form, causal and not, and forms that keep a block's keys in two parts:
# sequences, longest, seed of the lengths, heads, K/V heads, d_head, causal; form, orders, heads of a workgroup, parts of dK/dV.  5 rows
# before the first sequence and 11 behind the last.  Up to 64 sequences are ordered, more or one are taken from the end on.
ORDERED = [
    (60, 87, 9, 48, 6, 64, False, "S1", "oq", 4, 2),
    (60, 222, 9, 24, 12, 64, False, "S1", "okq", 2, 1),
    (33, 423, 0, 36, 12, 64, False, "S1", "oq", 1, 1),
    (64, 89, 4, 36, 12, 64, False, "W1", "oq", 1, 1),
    (64, 237, 0, 8, 8, 64, False, "W2", "o", 1, 1),
    (5, 225, 7, 32, 8, 64, False, "W4", "o", 4, 5),
    (64, 95, 4, 48, 12, 64, True, "S1", "oq", 4, 1),
    (64, 226, 7, 24, 12, 64, True, "S1", "okq", 2, 1),
    (64, 703, 7, 6, 6, 64, True, "S1", "okq", 1, 1),
    (60, 107, 3, 36, 12, 64, True, "W1", "oq", 1, 1),
    (5, 1182, 4, 12, 6, 64, True, "W2", "ok", 2, 3),
    (64, 180, 7, 8, 8, 64, True, "W2", "o", 1, 1),
    (3, 200, 4, 48, 6, 64, True, "W4", "o", 4, 10),
    (64, 62, 7, 48, 6, 128, False, "S1", "oq", 4, 2),
    (64, 127, 8, 24, 12, 128, False, "S1", "okq", 2, 1),
    (60, 87, 1, 36, 12, 128, False, "S1", "oq", 1, 1),
    (9, 495, 0, 16, 8, 128, False, "S2", "", 2, 1),
    (2, 1291, 7, 24, 8, 128, False, "S2", "ok", 1, 3),
    (64, 131, 4, 12, 12, 128, False, "W1", "ok", 1, 1),
    (9, 143, 7, 24, 8, 128, False, "W2", "o", 1, 3),
    (64, 122, 0, 4, 4, 128, False, "W4", "o", 1, 1),
    (60, 56, 9, 48, 12, 128, True, "S1", "oq", 4, 1),
    (60, 118, 9, 24, 12, 128, True, "S1", "okq", 2, 1),
    (64, 87, 6, 36, 12, 128, True, "S1", "oq", 1, 1),
    (3, 264, 4, 48, 12, 128, True, "S2", "", 4, 4),
    (33, 927, 4, 3, 1, 128, True, "S2", "ok", 1, 3),
    (64, 129, 4, 12, 12, 128, True, "W1", "ok", 1, 1),
    (5, 149, 4, 36, 12, 128, True, "W2", "o", 1, 3),
    (9, 86, 4, 24, 12, 128, True, "W4", "o", 2, 1),
    (80, 70, 1, 36, 12, 128, True, "S1", "oq", 1, 1),
    (90, 80, 1, 36, 12, 64, False, "W1", "oq", 1, 1),
    (1, 700, 1, 36, 36, 128, True, "W2", "o", 1, 1),
]
SHAPES = [c[:7] for c in ORDERED]
name = lambda c: f"{c[0]}upto{c[1]}-{c[3]}on{c[4]}-{c[5]}-{'causal' if c[6] else 'all'}"


@pytest.mark.parametrize("case", ORDERED, ids=name)
def test_the_batch_takes_the_form_it_is_for(case):
    n, longest, seed, h, kv, dh, causal, *want = case
    assert list(route("bf16", sum(ragged(n, longest, seed)) + 16, n, h, kv, dh, causal)) == want


def test_every_form_and_order_has_a_batch():
    met = set()
    for n, _, _, _, _, dh, causal, form, orders, heads, parts in ORDERED:
        if not 2 <= n <= 64:
            continue
        if "o" in orders:
            met.add((dh, causal, form, heads if form == "S1" else 0))
        if "k" in orders:
            met.add((dh, causal, "dK/dV", parts > 1))
        if "q" in orders:
            met.add((dh, causal, "dQ", heads))
    both = [(dh, causal) for dh in (64, 128) for causal in (False, True)]
    want = {(*b, "S1", heads) for b in both for heads in (1, 2, 4)} | {(*b, w, 0) for b in both for w in ("W1", "W2", "W4")}
    want |= {(128, causal, "S2", 0) for causal in (False, True)} | {(*b, "dQ", heads) for b in both for heads in (1, 2, 4)} | {(*b, "dK/dV", False) for b in both}
    assert want <= met, want - met


# The batches of test_gpu_packed_together.py's FORMS, in their order
@pytest.mark.parametrize("at,want", enumerate([("S1", 1), ("S2", 1), ("W1", 1), ("W2", 1), ("S1", 2), ("W2", 1), ("S1", 4), ("W1", 3), ("W1", 1), ("W2", 3), ("S2", 4), ("W1", 1)]))
def test_batches_of_the_other_tests(at, want):
    pytest.importorskip("torch")
    import test_gpu_packed_together as other
    lens, h, kv, dh, causal = other.FORMS[at]
    form, _, _, parts = route("bf16", sum(lens) + 16, len(lens), h, kv, dh, causal)
    assert (form, parts) == want


def test_short_batches_take_four_waves_to_a_block():
    for dh in (64, 128):
        for rows in (1, 30, 130, 333):
            assert route("bf16", rows, 1, 4, 2, dh, True)[0] == "W4"


@pytest.mark.parametrize("kw", [dict(dtype="f32"), dict(dh=32), dict(dh=16), dict(dh=8), dict(misaligned=True), dict(ld=1028)], ids=str)
def test_calls_with_fp32_products(kw):
    args = dict(dtype="bf16", rows=5000, n_seq=3, h=8, kv=4, dh=64, causal=True)
    assert route(**args)[0] != "fp32 products"
    form, orders, _, _ = route(**{**args, **kw})
    assert form == "fp32 products" and orders == ""
