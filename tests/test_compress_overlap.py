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
@pytest.mark.parametrize("other", SIZES)
def test_select_refuses_to_write_over_what_it_reads_or_writes(out, other):
    if out == other:
        return
    align = 16 if "ws" in (out, other) else 4
    for by in (0, (SIZES[other] - 1) // align * align, -((SIZES[out] - 1) // align * align)):
        assert _select(**{out: PLACES[other] + by}) == INVALID, by


def test_select_refuses_lists_over_pages():
    assert _select(pages=True, n_keep=PLACES["off"] + 4 * PAIRS * 2 - 4) == INVALID
