"""Compression of a growing cache: what its entry points refuse before anything touches a GPU, and the oracle's own pins (CPU only)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import compress as C
from test_step_refusals import AT, BAD_CACHES, _cache

INVALID, UNSUPPORTED = F.FAIRKV_EINVAL, F.FAIRKV_EUNSUPPORTED
ref = lambda c: ctypes.byref(c) if c else None


def _weights(c, q=AT, tree=None, n_new=None, len_=AT, lse=AT, weights=AT, out=AT, decay=1.0, n_slots=256, q_len=4, Hq=8, scale=0.1):
    return F.lib().fairkv_attn_weights(ref(c), q, tree, n_new, len_, lse, weights, out, decay, n_slots, q_len, Hq, scale, None)


def _select(c, budget=AT, shared=1, pool=1, sink=0, recent=0, weights=AT, len_=AT, keep=AT, max_keep=10, n_keep=AT, ws=AT, ws_bytes=1 << 40, n_slots=256, sel=True):
    s = F.fairkv_selection(budget, shared, pool, sink, recent)
    return F.lib().fairkv_select(ref(c), ref(s) if sel else None, weights, len_, keep, max_keep, n_keep, None, ws, ws_bytes, n_slots, None)


def _evict(c, into=None, keep=AT, max_keep=10, n_keep=2 * AT, len_=3 * AT, len_out=3 * AT, weights=None, out=None, n_slots=256):
    return F.lib().fairkv_evict(ref(c), ref(into), keep, max_keep, n_keep, len_, len_out, weights, out, None, n_slots, None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(kw, code):
    for call in (_weights, _select, _evict):
        assert call(_cache(**kw)) == code
    assert _evict(_cache(), into=_cache(**kw)) == code
    assert F.lib().fairkv_select_workspace_bytes(ref(_cache(**kw)), 1, 256) == 0


def test_no_cache():
    assert [call(None) for call in (_weights, _select, _evict)] == [INVALID] * 3
    assert F.lib().fairkv_select_workspace_bytes(None, 0, 256) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), INVALID), (dict(len_=None), INVALID), (dict(lse=None), INVALID), (dict(weights=None), INVALID), (dict(out=None), INVALID),
    (dict(q=AT + 8), INVALID), (dict(lse=AT + 2), INVALID), (dict(weights=AT + 1), INVALID), (dict(tree=AT + 4), INVALID),
    (dict(q_len=0), INVALID), (dict(q_len=65), UNSUPPORTED), (dict(Hq=0), INVALID), (dict(Hq=7), INVALID), (dict(Hq=34), UNSUPPORTED),
    (dict(n_slots=0), INVALID), (dict(n_slots=65537), UNSUPPORTED), (dict(scale=math.nan), INVALID), (dict(scale=3e38), INVALID),
    (dict(decay=math.inf), INVALID), (dict(decay=math.nan), INVALID),
    (dict(out=AT + 4), INVALID), (dict(out=AT + 396), INVALID), (dict(out=AT - 396), INVALID)])
def test_weights_refuse(kw, code):
    assert _weights(_cache(), **kw) == code


def test_weights_refuse_caches_of_fp32_and_too_many_queries():
    assert _weights(_cache(dtype=F.FAIRKV_F32)) == UNSUPPORTED
    assert _weights(_cache(B=1 << 17, Hkv=1), Hq=16, q_len=64) == INVALID
    assert _weights(_cache(dtype=F.FAIRKV_E4M3, n_scales=2, scales=[1.0, 3e38]), scale=1.0) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(sel=False), INVALID), (dict(budget=None), INVALID), (dict(weights=None), INVALID), (dict(len_=None), INVALID), (dict(keep=None), INVALID),
    (dict(n_keep=None), INVALID), (dict(max_keep=0), INVALID), (dict(n_slots=0), INVALID), (dict(n_slots=65537), UNSUPPORTED),
    (dict(shared=2), INVALID), (dict(shared=-1), INVALID), (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(pool=0), INVALID),
    (dict(pool=2), INVALID), (dict(pool=-3), INVALID), (dict(pool=65), UNSUPPORTED), (dict(ws=None), F.FAIRKV_EWORKSPACE),
    (dict(ws_bytes=15), F.FAIRKV_EWORKSPACE), (dict(ws=AT + 8), INVALID), (dict(weights=AT + 2), INVALID)])
def test_select_refuses(kw, code):
    assert _select(_cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(keep=None), INVALID), (dict(n_keep=None), INVALID), (dict(len_=None), INVALID), (dict(len_out=None), INVALID), (dict(max_keep=0), INVALID),
    (dict(n_slots=0), INVALID), (dict(n_slots=65537), UNSUPPORTED), (dict(weights=AT), INVALID), (dict(out=AT), INVALID),
    (dict(weights=AT, out=2 * AT), INVALID), (dict(weights=AT + 2, out=AT + 2), INVALID), (dict(len_out=2 * AT), INVALID), (dict(len_out=3 * AT + 4), INVALID),
    (dict(len_out=2 * AT + 12), INVALID)])
def test_evict_refuses(kw, code):
    assert _evict(_cache(), **kw) == code


@pytest.mark.parametrize("kw", [dict(B=3), dict(Hkv=1), dict(D=64), dict(dtype=F.FAIRKV_F32), dict(dtype=F.FAIRKV_E4M3, n_scales=1, scales=[1.0])])
def test_evict_refuses_a_cache_of_another_kind(kw):
    assert _evict(_cache(), into=_cache(**kw), len_out=AT) == INVALID


FAR = 1 << 40                                # addresses that are never read on the host
BYTES = 100 * 128 * 2                        # of the 100 rows of K


@pytest.mark.parametrize("kw", [dict(k=FAR, v=FAR + (1 << 30)), dict(k=FAR + BYTES - 16, v=FAR + (2 << 30)), dict(k=FAR + (2 << 30), v=FAR + 16),
                                dict(k=FAR + (2 << 30), v=FAR + (1 << 30) + BYTES - 16), dict(k=FAR + (1 << 30), v=FAR + (2 << 30))])
def test_evict_refuses_caches_that_share_rows(kw):
    c = _cache(k=FAR, v=FAR + (1 << 30))
    assert _evict(c, into=_cache(**kw), len_out=AT) == INVALID      # (the first is the cache itself: the same pool, and the same rows of it)


@pytest.mark.parametrize("into", [None, _cache(k=1 << 50, v=1 << 51)])
def test_evict_refuses_lists_whose_places_a_run_beyond_would_wrap(into):
    out = 3 * AT if into is None else AT
    for max_keep in (2**31 - 1, 2**31 - 65535):
        assert _evict(_cache(), into=into, max_keep=max_keep, len_out=out) == INVALID


def test_evict_refuses_weights_that_meet_those_that_are_read():
    c, other = _cache(k=FAR, v=FAR + (1 << 30)), _cache(k=FAR + (2 << 30), v=FAR + (3 << 30))
    for out in (8 * AT, 8 * AT + 396, 8 * AT - 396):
        assert _evict(c, into=other, len_out=AT, weights=8 * AT, out=out) == INVALID


def test_evict_refuses_other_scales():
    c = lambda x: _cache(dtype=F.FAIRKV_E4M3, n_scales=2, scales=[1.0, x])
    assert _evict(c(2.0), into=c(2.5), len_out=AT) == INVALID


def test_the_workspace_of_a_selection():
    need = lambda shared, n_slots=256, **kw: F.lib().fairkv_select_workspace_bytes(ctypes.byref(_cache(**kw)), shared, n_slots)
    small = need(0)
    assert 0 < small <= 4096 and need(1) == small                    # no group of 100 rows is a large one
    assert need(2) == need(-1) == need(0, 0) == need(0, 65537) == 0
    for shared in (0, 1):
        by_rows = [need(shared, n_rows=n) for n in (100, 7000, 20000, 1 << 20, 1 << 30)]
        assert by_rows == sorted(by_rows) and by_rows[-1] < (1 << 30) * 16
        assert _select(_cache(n_rows=1 << 20), shared=shared, ws_bytes=by_rows[3] - 1) == F.FAIRKV_EWORKSPACE
    # what pages say of the longest pair counts, not the size of the pool
    paged = dict(off=None, pages=AT, max_pages=64, page_rows=16, n_rows=1 << 24)
    assert need(0, **paged) == small and need(1, **paged) == small
    assert F.lib().fairkv_select_workspace_reset(None, 1 << 20, None) == INVALID
    assert F.lib().fairkv_select_workspace_reset(AT + 8, 1 << 20, None) == INVALID
    assert F.lib().fairkv_select_workspace_reset(AT, 100, None) == F.FAIRKV_EWORKSPACE


def test_more_pairs_than_a_launch_has():
    many = _cache(B=1 << 20, Hkv=64)
    assert _select(many, shared=0) == INVALID and _evict(many) == INVALID
    assert _select(_cache(B=(1 << 21) + 1, Hkv=1), shared=1) == INVALID


# ---- the oracle ----------------------------------------------------------------------------------------------
ROW = lambda p, t: 10 * p + t


def test_the_oracles_weights_sum_to_one_for_every_query():
    rng = np.random.default_rng(0)
    q, k, lens = rng.standard_normal((1, 2, 4, 8)), rng.standard_normal((20, 8)), np.array([[9, 6]])
    lse = np.zeros((1, 2, 4))
    for i in range(2):
        for g in range(4):
            p = g // 2
            seen = k[[ROW(p, t) for t in range(lens[0, p] - 1 + i)]]
            lse[0, i, g] = np.log(np.exp(0.3 * seen @ q[0, i, g]).sum())
    w = C.attn_weights(q, k, lens, lse, np.full(20, 5.0), 0.3, 0.0, [2], None, ROW)
    assert abs(w[:9].sum() - 4) < 1e-12 and abs(w[10:16].sum() - 4) < 1e-12
    assert (w[[9, 16, 17, 18, 19]] == 5).all()
    again = C.attn_weights(q, k, lens, lse, np.full(20, 5.0), 0.3, 0.5, [2], None, ROW)
    assert np.allclose(again[:9] - w[:9], [2.5] * 7 + [0, 0])


def test_the_oracles_selection():
    w = np.array([9, 1, 5, 5, 0, 7, 7, 2, 3, 1] + [6, 5, 5, 0, 0, 0, 0, 0, 0, 0], dtype=np.float64)
    lists, n = C.select(w, np.array([[10, 3]]), [5], True, 1, 1, 2, 10, ROW)      # protected: 0, 8, 9; 1, 2 and 0 of the other: 6 already
    assert lists == [[0, 8, 9], [0, 1, 2]] and n.tolist() == [[3, 3]]
    assert C.select(w, np.array([[10, 3]]), [5], True, 1, 0, 0, 10, ROW)[0] == [[0, 2, 5, 6], [0]]      # 9, 7, 7, 6, and of the 5s the first head's first
    assert C.select(w, np.array([[10, 3]]), [[3], [1]], False, 3, 0, 0, 10, ROW)[0] == [[0, 1, 4], [0]]
    assert C.select(w, np.array([[10, 3]]), [[3], [1]], False, 1, 0, 0, 2, ROW)[1].tolist() == [[-1, 1]]


def test_the_oracles_eviction():
    lens, keep = np.array([[6, 4]]), np.array([[[1, 4, 5], [2, 0, 0]]])
    assert C.evict(lens, keep, [[3, 1]], ROW)[1] == {0: 1, 1: 4, 2: 5, 10: 12}
    after, moves, alone = C.evict(lens, keep, [[3, 2]], ROW)
    assert after.tolist() == [3, 4] and alone == [1] and len(moves) == 3
    assert C.evict(lens, keep, [[3, 2]], ROW, lambda p, i: 100 + 10 * p + i, [[3, 3]])[1] == {100: 1, 101: 4, 102: 5, 110: 12, 111: 10}
