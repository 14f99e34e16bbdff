"""The workspace of the attention of a draft tree: what a call takes, by the sizes of the call (CPU only)."""
import ctypes

import numpy as np
import pytest

pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_step_refusals import AT, _cache, _tree


def _bytes(Hq, q_len, n_slots, **kw):
    return F.lib().fairkv_tree_workspace_bytes(ctypes.byref(_cache(**kw)), Hq, q_len, n_slots)


@pytest.mark.parametrize("n_slots", [1, 7, 40, 256, 1024])
@pytest.mark.parametrize("kw", [dict(n_rows=32768, B=1, Hkv=8), dict(n_rows=300, B=3, Hkv=2, D=64), dict(n_rows=1 << 22, B=64, Hkv=8),
                                dict(n_rows=1 << 30, B=64, Hkv=8, expected_rows=100000),
                                dict(n_rows=1 << 20, B=16, Hkv=8, off=None, pages=AT, max_pages=64, page_rows=16)])
def test_a_workspace_of_the_longest_draft_is_one_for_every_shorter_one(kw, n_slots):
    Hkv = kw["Hkv"]
    by_q = np.array([[_bytes(G * Hkv, q, n_slots, **kw) for q in range(1, 65)] for G in (1, 3, 8, 16)], dtype=np.int64)
    assert (by_q > 0).all() and (np.diff(by_q, axis=1) >= 0).all() and (np.diff(by_q, axis=0) >= 0).all()
    rows = [_bytes(8 * Hkv, 64, n_slots, **{**kw, "expected_rows": n}) for n in (1, 1000, 100000, 1 << 24, 1 << 40)]
    assert rows == sorted(rows)


def test_a_call_takes_a_workspace_of_a_longer_draft():
    kw = dict(n_rows=32768, B=1, Hkv=8)
    need = _bytes(64, 9, 256, **kw)
    assert _bytes(64, 8, 256, **kw) <= need
    assert _tree(_cache(**kw), Hq=64, q_len=9, ws_bytes=need - 1) == F.FAIRKV_EWORKSPACE
