"""A step over a growing cache: what its entry points refuse before anything touches a GPU, and the oracle's own pins (CPU only)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import step as S

AT = 4096      # stands for a device address: never read on the host


def _cache(**kw):
    c = dict(k=AT, v=AT, n_rows=100, off=AT, pages=None, cap=AT, max_pages=0, page_rows=0, B=2, Hkv=2, D=128, dtype=F.FAIRKV_BF16, n_scales=0)
    scales = kw.pop("scales", ())
    c.update(kw)
    c = F.fairkv_cache(**c)
    for i, x in enumerate(scales):
        c.k_scale[i] = c.v_scale[i] = x
    return c


def _append(c, r=None, q=AT, q_stride=1024, k_stride=256, q_out=2 * AT, q_len=4, Hq=8, dtype=F.FAIRKV_BF16, len_=AT, len_out=AT, k_new=AT, v_new=AT, v_stride=256):
    r = r or F.fairkv_rotation(eps=1e-6)
    return F.lib().fairkv_append_rotated(ctypes.byref(c) if c else None, ctypes.byref(r), q, q_stride, k_new, k_stride, v_new, v_stride, q_out, q_len, Hq,
                                         dtype, None, len_, len_out, None, None)


def _tree(c, q=AT, len_=AT, ws=AT, ws_bytes=1 << 40, n_slots=256, out=AT, q_len=4, Hq=8, out_dtype=F.FAIRKV_F32, scale=1.0, tree=None):
    return F.lib().fairkv_decode_attn_tree(ctypes.byref(c) if c else None, q, tree, None, len_, ws, ws_bytes, n_slots, out, None, q_len, Hq, out_dtype, scale, None)


def _accept(c, path=AT, n_path=AT, len_=AT, len_out=AT, q_len=4):
    return F.lib().fairkv_accept(ctypes.byref(c) if c else None, path, n_path, None, len_, len_out, q_len, None, None)


BAD_CACHES = [
    (dict(k=None), F.FAIRKV_EINVAL), (dict(v=None), F.FAIRKV_EINVAL), (dict(cap=None), F.FAIRKV_EINVAL), (dict(off=None), F.FAIRKV_EINVAL),
    (dict(pages=AT), F.FAIRKV_EINVAL), (dict(off=None, pages=AT), F.FAIRKV_EINVAL), (dict(off=None, pages=AT, max_pages=4, page_rows=8), F.FAIRKV_EINVAL),
    (dict(off=None, pages=AT, max_pages=4, page_rows=48), F.FAIRKV_EINVAL), (dict(off=None, pages=AT, max_pages=0, page_rows=16), F.FAIRKV_EINVAL),
    (dict(max_pages=4), F.FAIRKV_EINVAL), (dict(page_rows=16), F.FAIRKV_EINVAL), (dict(k=AT + 8), F.FAIRKV_EINVAL), (dict(v=AT + 2), F.FAIRKV_EINVAL),
    (dict(n_rows=-1), F.FAIRKV_EINVAL), (dict(expected_rows=-1), F.FAIRKV_EINVAL), (dict(B=0), F.FAIRKV_EINVAL), (dict(Hkv=0), F.FAIRKV_EINVAL), (dict(B=1 << 20, Hkv=1 << 11), F.FAIRKV_EINVAL),
    (dict(D=96), F.FAIRKV_EUNSUPPORTED), (dict(dtype=F.FAIRKV_BF16_VALU), F.FAIRKV_EUNSUPPORTED), (dict(n_scales=1, scales=[1.0]), F.FAIRKV_EINVAL),
    (dict(dtype=F.FAIRKV_E4M3), F.FAIRKV_EINVAL), (dict(dtype=F.FAIRKV_E4M3, n_scales=3, scales=[1.0] * 3), F.FAIRKV_EINVAL),
    (dict(dtype=F.FAIRKV_E4M3, n_scales=33, Hkv=33), F.FAIRKV_EUNSUPPORTED), (dict(dtype=F.FAIRKV_E4M3, n_scales=1, scales=[0.0]), F.FAIRKV_EINVAL),
    (dict(dtype=F.FAIRKV_E4M3, n_scales=2, scales=[1.0, math.inf]), F.FAIRKV_EINVAL), (dict(dtype=F.FAIRKV_E4M3, n_scales=1, scales=[math.nan]), F.FAIRKV_EINVAL)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(kw, code):
    for call in (_append, _tree, _accept):
        assert call(_cache(**kw)) == code
    assert F.lib().fairkv_tree_workspace_bytes(ctypes.byref(_cache(**kw)), 8, 4, 256) == 0


def test_no_cache():
    assert [call(None) for call in (_append, _tree, _accept)] == [F.FAIRKV_EINVAL] * 3
    assert F.lib().fairkv_tree_workspace_bytes(None, 8, 4, 256) == 0


def _rot(**kw):
    return F.fairkv_rotation(**{**dict(table=AT, pos=AT, eps=1e-6, n_pos=100, rot=64), **kw})


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), F.FAIRKV_EINVAL), (dict(k_new=None), F.FAIRKV_EINVAL), (dict(v_new=None), F.FAIRKV_EINVAL), (dict(q_out=None), F.FAIRKV_EINVAL),
    (dict(len_=None), F.FAIRKV_EINVAL), (dict(len_out=None), F.FAIRKV_EINVAL), (dict(q_len=0), F.FAIRKV_EINVAL), (dict(Hq=0), F.FAIRKV_EINVAL),
    (dict(q_len=65), F.FAIRKV_EUNSUPPORTED), (dict(dtype=F.FAIRKV_F32), F.FAIRKV_EUNSUPPORTED), (dict(dtype=F.FAIRKV_E4M3), F.FAIRKV_EUNSUPPORTED),
    (dict(q_stride=1016), F.FAIRKV_EINVAL), (dict(q_stride=1028), F.FAIRKV_EINVAL), (dict(k_stride=248), F.FAIRKV_EINVAL), (dict(v_stride=260), F.FAIRKV_EINVAL),
    (dict(q=AT + 4), F.FAIRKV_EINVAL), (dict(k_new=AT + 8), F.FAIRKV_EINVAL), (dict(v_new=AT + 2), F.FAIRKV_EINVAL), (dict(q_out=AT + 2), F.FAIRKV_EINVAL),
    (dict(q_out=AT, q_stride=1280), F.FAIRKV_EINVAL), (dict(k_new=2 * AT), F.FAIRKV_EINVAL), (dict(v_new=2 * AT), F.FAIRKV_EINVAL),
    (dict(r=_rot(pos=None)), F.FAIRKV_EINVAL), (dict(r=_rot(n_pos=0)), F.FAIRKV_EINVAL), (dict(r=_rot(rot=0)), F.FAIRKV_EINVAL), (dict(r=_rot(rot=8)), F.FAIRKV_EINVAL),
    (dict(r=_rot(rot=40)), F.FAIRKV_EINVAL), (dict(r=_rot(rot=144)), F.FAIRKV_EINVAL), (dict(r=_rot(table=AT + 4)), F.FAIRKV_EINVAL),
    (dict(r=_rot(q_norm=AT, eps=-1.0)), F.FAIRKV_EINVAL), (dict(r=_rot(k_norm=AT, eps=math.nan)), F.FAIRKV_EINVAL)])
def test_append_refuses(kw, code):
    assert _append(_cache(), **kw) == code


def test_append_of_fp32_rows_wants_an_fp32_cache():
    assert _append(_cache(dtype=F.FAIRKV_F32)) == F.FAIRKV_EUNSUPPORTED
    assert _append(_cache(dtype=F.FAIRKV_E4M3, n_scales=1, scales=[1.0]), dtype=F.FAIRKV_F32) == F.FAIRKV_EUNSUPPORTED


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), F.FAIRKV_EINVAL), (dict(len_=None), F.FAIRKV_EINVAL), (dict(out=None), F.FAIRKV_EINVAL), (dict(ws=None), F.FAIRKV_EWORKSPACE),
    (dict(q_len=0), F.FAIRKV_EINVAL), (dict(Hq=7), F.FAIRKV_EINVAL), (dict(Hq=0), F.FAIRKV_EINVAL), (dict(n_slots=0), F.FAIRKV_EINVAL),
    (dict(q_len=65), F.FAIRKV_EUNSUPPORTED), (dict(Hq=34), F.FAIRKV_EUNSUPPORTED), (dict(n_slots=65537), F.FAIRKV_EUNSUPPORTED),
    (dict(out_dtype=F.FAIRKV_E4M3), F.FAIRKV_EUNSUPPORTED), (dict(scale=math.inf), F.FAIRKV_EINVAL), (dict(scale=math.nan), F.FAIRKV_EINVAL),
    (dict(q=AT + 8), F.FAIRKV_EINVAL), (dict(out=AT + 8), F.FAIRKV_EINVAL), (dict(ws=AT + 8), F.FAIRKV_EINVAL), (dict(tree=AT + 4), F.FAIRKV_EINVAL),
    (dict(ws_bytes=0), F.FAIRKV_EWORKSPACE)])
def test_tree_refuses(kw, code):
    assert _tree(_cache(), **kw) == code


def test_tree_refuses_more_than_it_can_address_and_an_fp32_cache():
    assert _tree(_cache(B=1 << 16, Hkv=4), Hq=64, q_len=64) == F.FAIRKV_EINVAL
    assert _tree(_cache(dtype=F.FAIRKV_F32)) == F.FAIRKV_EUNSUPPORTED


@pytest.mark.parametrize("scale,k_scale", [(3e38, 1.0), (1.0, 3e38), (-1e30, 1e30)])
def test_tree_refuses_factors_that_are_no_numbers(scale, k_scale):
    assert _tree(_cache(dtype=F.FAIRKV_E4M3, n_scales=2, scales=[1.0, k_scale]), scale=scale) == F.FAIRKV_EINVAL
    if k_scale == 1.0:
        assert _tree(_cache(), scale=scale) == F.FAIRKV_EINVAL


def test_a_scale_without_a_reciprocal_is_refused():
    c = _cache(dtype=F.FAIRKV_E4M3, n_scales=1, scales=[1e-45])
    assert [call(c) for call in (_append, _tree, _accept)] == [F.FAIRKV_EINVAL] * 3


def test_tree_workspace_of_caches_of_any_size():
    """Rows, pages and pairs whose products leave 64 bits: what a cache of so many rows takes, whatever its pages."""
    L, n = F.lib(), 1 << 62
    packed = L.fairkv_tree_workspace_bytes(ctypes.byref(_cache(n_rows=n, B=1 << 12, Hkv=8)), 64, 64, 256)
    paged = _cache(n_rows=n, off=None, pages=AT, max_pages=(1 << 31) - 1, page_rows=1 << 30, B=1 << 12, Hkv=8)
    assert 0 < L.fairkv_tree_workspace_bytes(ctypes.byref(paged), 64, 64, 256) == packed
    few = _cache(n_rows=n, off=None, pages=AT, max_pages=1, page_rows=16, B=1, Hkv=8)
    assert 0 < L.fairkv_tree_workspace_bytes(ctypes.byref(few), 64, 8, 256) < packed


def test_expected_rows_decide_how_columns_are_dealt_and_never_beyond_the_cache():
    L, size = F.lib(), lambda **kw: F.lib().fairkv_tree_workspace_bytes(ctypes.byref(_cache(B=4, Hkv=8, **kw)), 64, 24, 256)
    assert size(n_rows=1 << 24, expected_rows=20000) == size(n_rows=20000) < size(n_rows=1 << 24)
    assert size(n_rows=20000, expected_rows=1 << 40) == size(n_rows=20000)
    assert ctypes.sizeof(F.fairkv_cache) == 344


def test_tree_workspace():
    L, c = F.lib(), _cache()
    for Hq, q_len, n_slots in ((8, 4, 256), (2, 1, 1), (32, 64, 256), (6, 33, 7)):
        need = L.fairkv_tree_workspace_bytes(ctypes.byref(c), Hq, q_len, n_slots)
        assert need > 0
        assert _tree(c, Hq=Hq, q_len=q_len, n_slots=n_slots, ws_bytes=need - 1) == F.FAIRKV_EWORKSPACE


def test_tree_workspace_reset_and_its_counters():
    L = F.lib()
    assert [L.fairkv_tree_counter_bytes(n) for n in (0, -1, 65537)] == [0, 0, 0]
    assert 0 < L.fairkv_tree_counter_bytes(1) <= L.fairkv_tree_counter_bytes(256) < L.fairkv_tree_workspace_bytes(ctypes.byref(_cache()), 8, 4, 256)
    for args, code in (((None, 1 << 30, 256), F.FAIRKV_EINVAL), ((AT + 4, 1 << 30, 256), F.FAIRKV_EINVAL), ((AT, 1 << 30, 0), F.FAIRKV_EINVAL),
                       ((AT, F.fairkv_tree_counter_bytes(256) - 1, 256), F.FAIRKV_EWORKSPACE)):
        assert L.fairkv_tree_workspace_reset(*args, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(path=None), F.FAIRKV_EINVAL), (dict(n_path=None), F.FAIRKV_EINVAL), (dict(len_=None), F.FAIRKV_EINVAL), (dict(len_out=None), F.FAIRKV_EINVAL),
    (dict(q_len=0), F.FAIRKV_EINVAL), (dict(q_len=65), F.FAIRKV_EUNSUPPORTED)])
def test_accept_refuses(kw, code):
    assert _accept(_cache(), **kw) == code


def test_a_cache_is_checked_when_it_is_made():
    k, cap, off = torch.zeros(8, 64, dtype=torch.bfloat16), torch.ones(1, 2, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int64)
    pages = torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        F.Cache(k, k, cap, off=off)
    for kw in (dict(), dict(off=off, pages=pages, page_rows=16), dict(pages=pages), dict(off=off, page_rows=16), dict(off=off.int()),
               dict(pages=pages.long(), page_rows=16), dict(pages=pages[:1], page_rows=16), dict(off=off[:, :1])):
        with pytest.raises(ValueError):
            F.Cache(k, k, cap, **kw)
    with pytest.raises(TypeError):
        F.Cache(k.half(), k.half(), cap, off=off)
    with pytest.raises(TypeError):
        F.Cache(k, k.float(), cap, off=off)
    with pytest.raises(ValueError):
        F.Cache(k, k[:4], cap, off=off)


def test_a_call_refuses_tensors_that_are_not_on_the_caches_gpu():
    class Host:      # a cache whose tensors are never looked at
        struct = _cache()
        address, device, n_slots = ctypes.addressof(struct), 0, 256
    n = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, kv = torch.zeros(2, 4, 8, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        F.fairkv_append_rotated(Host, n(2, 2), q, kv, kv, q.clone())
    with pytest.raises(ValueError, match="device"):
        F.fairkv_decode_attn_tree(Host, n(2, 2), q, n(1), q.clone(), None, 1.0)
    with pytest.raises(ValueError, match="device"):
        F.fairkv_accept(Host, n(2, 2), n(2, 4), n(2))
    with pytest.raises(TypeError):
        F.fairkv_accept(Host, None, n(2, 4), n(2))


# ---- the oracle ----------------------------------------------------------------------------------------
def test_oracle_rotation_is_a_product_of_complex_numbers_and_keeps_lengths():
    rng = np.random.default_rng(0)
    x, angle = rng.standard_normal((3, 2, 64)), rng.uniform(0, 6, (10, 16))
    table, pos = np.concatenate([np.cos(angle), np.sin(angle)], 1), np.array([0, 9, 4])
    for pairs in (False, True):
        y = S.turned(x, None, 0.0, table, pos, pairs)
        a, b = (slice(0, 32, 2), slice(1, 32, 2)) if pairs else (slice(0, 16), slice(16, 32))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * angle[pos])[:, None]
        np.testing.assert_allclose(y[..., a] + 1j * y[..., b], z, atol=1e-14)
        np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
    y = S.turned(x, np.ones(64), 0.0, None, None, False)
    np.testing.assert_allclose((y ** 2).mean(-1), 1.0)


def test_oracle_attention_of_a_chain_is_that_of_shorter_caches():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((40, 64)), rng.standard_normal((40, 64)), rng.standard_normal((1, 3, 2, 64))
    row = lambda p, t: S.row_of(p, t, 40, off=[5])
    out, lse, *_ = S.attend(q, k, v, [[20]], [3], lambda b, i, j: j <= i, 0.3, 1, row)
    for i in range(3):
        one, l1, *_ = S.attend(q[:, i:i + 1], k, v, [[18 + i]], [1], lambda *_: True, 0.3, 1, row)
        np.testing.assert_allclose(out[:, i], one[:, 0])
        np.testing.assert_allclose(lse[:, i], l1[:, 0])


def test_oracle_rows_and_what_is_left_alone():
    pages = np.array([[2, 0], [1, 9]])
    assert [S.row_of(0, t, 48, pages=pages, page_rows=16) for t in (0, 15, 16, 32)] == [32, 47, 0, None]
    assert S.row_of(1, 16, 48, pages=pages, page_rows=16) is None
    row = lambda p, t: S.row_of(p, t, 48, pages=pages, page_rows=16)
    lens, rows, alone = S.append([15, 15], [32, 32], [2], 2, row, [[True, True]])
    assert lens.tolist() == [17, 15] and rows == {(0, 0): 47, (0, 1): 0} and alone == [1]
    lens, moves, alone = S.accept([17, 17], [[1, 0]], [1], [2], 2, row)
    assert lens.tolist() == [16, 17] and moves == {47: 0} and alone == [1]
