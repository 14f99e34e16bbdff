"""Queries of an append that would be written over what is still read are refused (CPU only)."""
import pytest

pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_step_refusals import _append, _cache

FAR = 1 << 40                                # addresses that are never read on the host
Q, KV = 8 * 128 * 2, 2 * 128 * 2             # bytes of a token's heads; 2 x 4 tokens
N = 8


@pytest.mark.parametrize("where", [
    dict(q=FAR, q_out=FAR + 16), dict(q=FAR + 16, q_out=FAR), dict(q=FAR, q_out=FAR + N * Q - 16),                         # a part of q
    dict(k_new=FAR, q_out=FAR + N * KV - 16), dict(k_new=FAR + N * Q - 16, q_out=FAR), dict(v_new=FAR + 16, q_out=FAR),    # of k_new, v_new
    dict(q=FAR, q_stride=1536, q_out=FAR + Q), dict(k_new=FAR, k_stride=1536, q_out=FAR + KV),                             # between the tokens of a projection
    dict(v_new=FAR, v_stride=1 << 62, q_out=FAR + (1 << 50)), dict(q=FAR, q_stride=1536, q_out=FAR)])
def test_queries_over_what_is_read(where):
    apart = {"q": FAR + (1 << 30), "k_new": FAR + (2 << 30), "v_new": FAR + (3 << 30)}
    assert _append(_cache(), **{**apart, **where}) == F.FAIRKV_EINVAL
