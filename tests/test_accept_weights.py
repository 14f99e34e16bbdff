"""An accept that moves weights: what it refuses before anything touches a GPU (CPU only)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_step_refusals import AT, BAD_CACHES, _cache


def _accept(c, weights=AT, path=AT, n_path=AT, len_=AT, len_out=AT, q_len=4):
    return F.lib().fairkv_accept_weights(ctypes.byref(c) if c else None, weights, path, n_path, None, len_, len_out, q_len, None, None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_a_bad_cache(kw, code):
    assert _accept(_cache(**kw)) == code and _accept(None) == F.FAIRKV_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(weights=AT + 2), F.FAIRKV_EINVAL), (dict(path=None), F.FAIRKV_EINVAL), (dict(n_path=None), F.FAIRKV_EINVAL), (dict(len_=None), F.FAIRKV_EINVAL),
    (dict(len_out=None), F.FAIRKV_EINVAL), (dict(q_len=0), F.FAIRKV_EINVAL), (dict(q_len=65), F.FAIRKV_EUNSUPPORTED)])
def test_refusals(kw, code):
    assert _accept(_cache(), **kw) == code


def test_weights_on_the_host():
    class Host:      # a cache whose tensors are never looked at
        struct = _cache()
        address, device, n_slots = ctypes.addressof(struct), 0, 256
    n = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises((ValueError, TypeError)):
        F.fairkv_accept(Host, n(2, 2), n(2, 4), n(2), weights=torch.zeros(100))
