"""The largest calls of a step over a growing cache: what no launch can hold is refused before one is made (CPU only)."""
import pytest

pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_step_refusals import _accept, _append, _cache


@pytest.mark.parametrize("dtype,D", [(F.FAIRKV_BF16, 128), (F.FAIRKV_F32, 128), (F.FAIRKV_F32, 64)])
def test_more_pairs_than_a_launch_has_workgroups(dtype, D):
    many = _cache(B=1 << 21, Hkv=16, dtype=dtype, D=D)
    assert _accept(many, q_len=64) == F.FAIRKV_EINVAL
    assert _append(many, q_len=64, Hq=16, dtype=dtype, q_stride=16 * D, k_stride=16 * D, v_stride=16 * D) == F.FAIRKV_EINVAL


def test_more_tokens_than_a_launch_has_workgroups():
    assert _append(_cache(B=(1 << 24) + (1 << 23), Hkv=1), q_len=64, Hq=1, q_stride=128, k_stride=128, v_stride=128) == F.FAIRKV_EINVAL
