"""The widest rows that the embedding on packed sequences takes: its limits are counted in 64 bits.  Decided on the host, so without a GPU."""
import pytest

from paper_2410_07192_amd import binding as pf

P = 1 << 20      # an aligned address nothing reads: every call here is refused
WIDEST = 2 ** 31 - 8


@pytest.mark.parametrize("tokens,d", [(17, WIDEST), (1 << 26, WIDEST), ((1 << 26) // 2 + 1, 520), (33, 2 ** 30 + 8)])
def test_rows_past_the_limit_are_refused(tokens, d):
    """tokens * ceil(d / 512) of more than 2^26."""
    calls = [lambda: pf.pf_op_embed_packed(pf.PF_DTYPE_BF16, P, P, None, None, 0, 1.0, P, tokens, 8, d, 10),
             lambda: pf.pf_op_embed_packed_bwd_workspace(tokens, 8, d, 10),
             lambda: pf.pf_op_embed_packed_bwd(pf.PF_DTYPE_BF16, P, P, None, 0, 1.0, P, None, 0, P, 1 << 60, tokens, 8, d, 10)]
    for call in calls:
        with pytest.raises(pf.PipeFillError) as e:
            call()
        assert e.value.code == pf.PF_ERR_ARG


@pytest.mark.parametrize("tokens,d", [(16, WIDEST), (1, WIDEST), (1 << 26, 512), (31, 2 ** 30 + 8)])
def test_the_workspace_of_the_widest_rows(tokens, d):
    """Two partial sums of d floats for tokens and for positions, for every share of at most 16 rows."""
    n = pf.pf_op_embed_packed_bwd_workspace(tokens, 8, d, 10)
    assert n >= 2 * 2 * 4 * d * ((tokens + 15) // 16)
