"""Compression of a growing cache: calls that would write over what they read are refused before anything touches a GPU (CPU only)."""
import ctypes

import pytest

pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_step_refusals import _cache

INVALID = F.FAIRKV_EINVAL
AT = 1 << 40                                 # addresses, far apart, that are never read on the host
PLACES = {name: AT + (i << 30) for i, name in enumerate(("k", "v", "off", "cap", "weights", "len", "budget", "keep", "n_keep", "bad", "ws", "len_out", "weights_out"))}
ROWS, PAIRS, MOST, WS = 100, 4, 10, 1 << 20


def _select(pages=False, shared=1, **places):
    p = dict(PLACES, **places)
    where = dict(off=None, pages=p["off"], max_pages=2, page_rows=16) if pages else dict(off=p["off"])
    c = _cache(k=p["k"], v=p["v"], cap=p["cap"], n_rows=ROWS, **where)
    s = F.fairkv_selection(p["budget"], shared, 1, 0, 0)
    return F.lib().fairkv_select(ctypes.byref(c), ctypes.byref(s), p["weights"], p["len"], p["keep"], MOST, p["n_keep"], p["bad"], p["ws"], WS, 256, None)


SIZES = {"weights": 4 * ROWS, "len": 4 * PAIRS, "budget": 4 * 2, "off": 8 * PAIRS, "keep": 4 * PAIRS * MOST, "n_keep": 4 * PAIRS, "bad": 4, "ws": WS}
WRITTEN = ("keep", "n_keep", "bad", "ws")


@pytest.mark.parametrize("out", WRITTEN)
@pytest.mark.parametrize("other", ("weights", "len", "budget", "off") + WRITTEN)
def test_select_refuses_to_write_over_what_it_reads_or_writes(out, other):
    if out == other:
        return
    align = 16 if "ws" in (out, other) else 4
    for by in (0, (SIZES[other] - 1) // align * align, -((SIZES[out] - 1) // align * align)):
        assert _select(**{out: PLACES[other] + by}) == INVALID, by


def test_select_refuses_lists_over_pages():
    assert _select(pages=True, n_keep=PLACES["off"] + 4 * PAIRS * 2 - 4) == INVALID


def _evict(other_cache=False, pages=False, **places):
    p = dict(PLACES, **places)
    where = dict(off=None, pages=p["off"], max_pages=2, page_rows=16) if pages else dict(off=p["off"])
    c = _cache(k=p["k"], v=p["v"], cap=p["cap"], n_rows=ROWS, **where)
    into = _cache(k=p["k"] + (1 << 38), v=p["v"] + (1 << 38), cap=p["into_cap"], off=p["into_off"], n_rows=ROWS) if other_cache else None
    return F.lib().fairkv_evict(ctypes.byref(c), ctypes.byref(into) if into else None, p["keep"], MOST, p["n_keep"], p["len"], p["len_out"], p["weights"],
                                p["weights_out"] if other_cache else p["weights"], p["bad"], 256, None)


PLACES.update(into_off=AT + (60 << 30), into_cap=AT + (61 << 30))
SIZES.update(len_out=4 * PAIRS, weights_out=4 * ROWS, into_off=8 * PAIRS, into_cap=4 * PAIRS)


@pytest.mark.parametrize("other_cache", [False, True])
@pytest.mark.parametrize("out", ["len_out", "bad", "weights_out"])
@pytest.mark.parametrize("other", ["keep", "n_keep", "off", "into_off", "into_cap", "len_out", "bad", "weights_out"])
def test_evict_refuses_to_write_over_what_it_reads_or_writes(out, other, other_cache):
    if out == other or (not other_cache and (other.startswith("into") or "weights_out" in (out, other))):
        return
    for by in (0, (SIZES[other] - 1) // 4 * 4, -((SIZES[out] - 1) // 4 * 4)):
        assert _evict(other_cache, **{out: PLACES[other] + by}) == INVALID, by


def test_evict_in_place_refuses_weights_over_lists_and_lengths_over_pages():
    for name in ("keep", "n_keep", "off", "len_out", "bad"):
        assert _evict(weights=PLACES[name]) == INVALID, name
    assert _evict(pages=True, len_out=PLACES["off"] + 4 * PAIRS * 2 - 4) == INVALID
    assert _evict(pages=True, bad=PLACES["off"] + 4) == INVALID


@pytest.mark.parametrize("dtype,row", [(F.FAIRKV_BF16, 256), (F.FAIRKV_F32, 512)])
def test_evict_refuses_keys_that_meet_values(dtype, row):
    """In place, or in the cache that rows go to; where they come from does not matter."""
    p = {name: at + (1 << 39) for name, at in PLACES.items()}
    cache = lambda k, v: ctypes.byref(_cache(k=k, v=v, cap=p["cap"], off=p["off"], n_rows=ROWS, dtype=dtype))
    call = lambda c, into: F.lib().fairkv_evict(c, into, p["keep"], MOST, p["n_keep"], p["len"], p["len_out"], None, None, None, 256, None)
    for by in (0, 16, row * ROWS - 16, -(row * ROWS - 16)):
        assert call(cache(AT, AT + by), None) == INVALID, by
        assert call(cache(AT + (1 << 36), AT + (1 << 37)), cache(AT, AT + by)) == INVALID, by
