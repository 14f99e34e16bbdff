"""A step over a growing cache on the GPU against the oracle: append with norms and rotation, attention of a draft tree, accept, and the
three in a row.

Tolerances, by what is rounded (a bf16 number is off by at most 2^-8 of itself, E4M3 by 2^-4 or 2^-10 near zero, fp32 by 2^-24):
  turned heads  16 fp32 roundings on the way (8 + 4 of the sum of squares, of which the root takes half, root, quotient, two products, two of the
                rotation) of terms no larger than |a| + |b|: 2^-19 (|a| + |b|) with room for the root's and the quotient's own, and the type's rounding.
  scores        D products summed in fp32: at most D 2^-24 of S = scale sum_d |q_d k_d|, 2^-23 of the rest; a weight is off by as much of
                itself, and twice that against the sum of the weights.
  weights       two bf16 parts: 2^-16; one (bf16 outputs of many columns): 2^-8.  out is a mean of rows: off by at most that of max |v|.
  sums          of n weights: n 2^-24."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import step as S

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "kv8": torch.float8_e4m3fn}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24, "kv8": 2.0 ** -4}
I32 = lambda x: torch.as_tensor(np.ascontiguousarray(x, dtype=np.int32), device=DEV)


def _bits(x):
    return x.view(torch.uint8)


class Setup:
    """A cache with lengths `lens` [B][Hkv] and `room` more rows a pair, filled with finite numbers, packed or in pages in no order."""

    def __init__(self, lens, room, D, dtype="bf16", page=0, seed=0, scales=None, pool=0):
        self.lens_h = np.asarray(lens, dtype=np.int64)
        self.B, self.Hkv = self.lens_h.shape
        self.D, self.dtype, self.page = D, dtype, page
        rng = np.random.default_rng(seed)
        cap = np.maximum(self.lens_h, 0) + room
        self.off = self.pages = None
        if page:
            need = -(-cap // page).reshape(-1)
            n_pages = int(need.sum()) + 3 + pool
            order = rng.permutation(n_pages)[:need.sum()]
            self.pages = np.full((need.size, max(int(need.max()), 1)), -7, dtype=np.int32)
            self.pages[np.arange(self.pages.shape[1])[None, :] < need[:, None]] = order
            self.n_rows = n_pages * page
        else:
            gaps = cap.reshape(-1) + rng.integers(0, 3, cap.size)
            self.off = np.concatenate([[0], np.cumsum(gaps)[:-1]]) + 1
            self.n_rows = int(gaps.sum()) + 2
        self.cap_h = cap
        g = torch.Generator().manual_seed(seed)
        rows = lambda: torch.randn(self.n_rows, D, generator=g).to(torch.bfloat16 if dtype == "kv8" else TYPES[dtype])
        self.k, self.v = (x.to(TYPES[dtype]).to(DEV) for x in (rows() * 8 if dtype == "kv8" else rows(), rows()))
        self.ks = self.vs = np.ones(self.Hkv)
        if dtype == "kv8" and scales:
            self.ks, self.vs = (np.linspace(a, b, self.Hkv, dtype=np.float32) for a, b in ((0.02, 0.05), (0.5, 0.25)))
        self.make()

    def make(self):
        kw = dict(k_scale=self.ks.tolist(), v_scale=self.vs.tolist()) if self.dtype == "kv8" else {}
        self.cache = F.Cache(self.k, self.v, I32(self.cap_h), **kw,
                             **(dict(pages=I32(self.pages), page_rows=self.page) if self.page else
                                dict(off=torch.as_tensor(self.off.reshape(self.B, self.Hkv), device=DEV))))
        self.lens = I32(self.lens_h)
        return self

    def row(self, pair, t):
        return S.row_of(pair, t, self.n_rows, None if self.page else self.off, self.pages, self.page)

    def numbers(self):
        """k and v as the numbers in the cache, without the scales of an 8-bit one."""
        return self.k.float().cpu().numpy().astype(np.float64), self.v.float().cpu().numpy().astype(np.float64)


# ---- append ----------------------------------------------------------------------------------------------
def _new(s, q_len, Hq, seed, fused, flat=False):
    g = torch.Generator().manual_seed(seed + 77)
    dt = torch.float32 if s.dtype == "f32" else torch.bfloat16
    x = torch.randn(s.B, q_len, Hq + 2 * s.Hkv, s.D, generator=g).to(dt).to(DEV)
    parts = x.split([Hq, s.Hkv, s.Hkv], dim=2)
    parts = parts if fused else [p.contiguous() for p in parts]
    return [p[:, 0] for p in parts] if flat else list(parts)


def _table(n_pos, rot, seed):
    angle = np.random.default_rng(seed + 5).uniform(-7, 7, (n_pos, rot // 2))
    return torch.tensor(np.concatenate([np.cos(angle), np.sin(angle)], 1), dtype=torch.float32, device=DEV)


def _check_append(s, q, k_new, v_new, q_out, before, q_before, lens_out, bad, kw, n_new):
    table, pos = kw.get("table"), kw.get("pos")
    host = lambda t: None if t is None else t.float().cpu().numpy().astype(np.float64)
    q4, k4, v4 = (x if x.dim() == 4 else x[:, None] for x in (q, k_new, v_new))
    n = q4.shape[1]
    pos_h = np.zeros((s.B, n), dtype=np.int64) if pos is None else pos.cpu().numpy().reshape(s.B, n)
    ok_pos = np.ones((s.B, n), dtype=bool) if table is None else (pos_h >= 0) & (pos_h < table.shape[0])
    nn = np.clip(n_new, 0, n)
    lens, rows, alone = S.append(s.lens_h, s.cap_h, nn, s.Hkv, s.row, ok_pos)
    assert lens_out.cpu().numpy().reshape(-1).tolist() == lens.tolist()
    left = [(b, i) for b in range(s.B) for i in range(nn[b]) if not ok_pos[b, i]]
    if bad is not None:
        assert int(bad) == len(alone) + len(left)
    safe = np.where(ok_pos, pos_h, 0)
    turn = lambda x, w: S.turned(host(x), host(w), kw.get("eps", 1e-6), host(table), safe, kw.get("pairs", False))

    def slack(x, w):      # 2^-19 of |a| + |b| of the rotation's pairs; the whole row's largest stands for both
        y = S.turned(host(x), host(w), kw.get("eps", 1e-6), None, None, False)
        return 2.0 ** -19 * 2 * np.abs(y).max(-1, keepdims=True)

    want, got = turn(q4, kw.get("q_norm")), host(q_out).reshape(q4.shape)
    plain = "f32" if s.dtype == "f32" else "bf16"
    tol = HALF[plain] * np.abs(want) + slack(q4, kw.get("q_norm"))
    for b in range(s.B):
        for i in range(n):
            if i < nn[b] and ok_pos[b, i]:
                assert (np.abs(got[b, i] - want[b, i]) <= tol[b, i]).all(), (b, i)
            else:
                np.testing.assert_array_equal(got[b, i], host(q_before).reshape(q4.shape)[b, i])
    k_want, v_want, k_slack = turn(k4, kw.get("k_norm")), host(v4), slack(k4, kw.get("k_norm"))
    k_got, v_got = s.numbers()
    touched = np.zeros(s.n_rows, dtype=bool)
    for (p, i), r in rows.items():
        b, h = divmod(p, s.Hkv)
        touched[r] = True
        for got_row, w, sl, sc in ((k_got[r], k_want[b, i, h], k_slack[b, i, h], s.ks[h]), (v_got[r], v_want[b, i, h], 0.0, s.vs[h])):
            if s.dtype == "kv8":
                w = np.clip(w / sc, -448, 448)
                t = 2.0 ** -4 * np.abs(w) * (1 + 2.0 ** -20) + 2.0 ** -10 + sl / sc
            else:
                t = HALF[s.dtype] * np.abs(w) + sl
            assert (np.abs(got_row - w) <= t).all(), (p, i)
    keep = torch.as_tensor(~touched, device=DEV)
    assert torch.equal(_bits(s.k)[keep], _bits(before[0])[keep]) and torch.equal(_bits(s.v)[keep], _bits(before[1])[keep])


def _run_append(s, q_len, Hq, seed=0, fused=False, flat=False, n_new=None, lens_out=True, in_place=False, **kw):
    q, k_new, v_new = _new(s, q_len, Hq, seed, fused, flat)
    q_in = q.clone()
    q_out = q if in_place else torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    before, q_before = (s.k.clone(), s.v.clone()), q_out.clone()
    out = torch.full_like(s.lens, -5) if lens_out else None
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    F.fairkv_append_rotated(s.cache, s.lens, q, k_new, v_new, q_out, n_new=None if n_new is None else I32(n_new), lens_out=out, bad=bad, **kw)
    torch.cuda.synchronize()
    _check_append(s, q_in, k_new, v_new, q_out, before, q_before, out if lens_out else s.lens, bad, kw, np.full(s.B, q_len) if n_new is None else np.asarray(n_new))


LENS = [[0, 1, 17], [64, 5, 31], [16, 47, 100]]


@pytest.mark.parametrize("dtype", ["bf16", "f32", "kv8"])
@pytest.mark.parametrize("D,Hq,q_len,page,rot,pairs,norm,fused", [
    (128, 24, 1, 0, 128, False, True, True), (64, 3, 1, 16, 64, True, False, False), (128, 3, 5, 32, 64, False, True, False),
    (64, 21, 16, 0, 16, True, True, True), (128, 48, 17, 16, 128, True, True, True), (64, 9, 33, 64, 32, False, False, True),
    (128, 6, 64, 0, 48, False, True, True), (64, 51, 64, 16, 64, False, True, False), (128, 3, 2, 0, 0, False, True, False), (64, 12, 7, 128, 0, False, False, True)])
def test_append(dtype, D, Hq, q_len, page, rot, pairs, norm, fused):
    s = Setup(LENS, q_len + 1, D, dtype, page, seed=D + q_len, scales=True)
    kw = {}
    if rot:
        kw.update(table=_table(50, rot, q_len), pos=I32(np.random.default_rng(q_len).integers(0, 50, (3, q_len))), pairs=pairs)
    if norm:
        kw.update({n: torch.tensor(1 + 0.3 * np.random.default_rng(i).standard_normal(D), dtype=torch.float32, device=DEV) for i, n in enumerate(("q_norm", "k_norm"))}, eps=1e-5)
    _run_append(s, q_len, Hq, fused=fused, **kw)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("lens_out", [False, True])
def test_append_ragged_in_place_and_flat(page, lens_out):
    s = Setup(np.arange(2 * 70).reshape(70, 2) % 40, 8, 128, page=page, seed=3)
    _run_append(s, 8, 4, n_new=np.random.default_rng(0).integers(-2, 12, 70), lens_out=lens_out, in_place=True, table=_table(9, 128, 0),
                pos=I32(np.random.default_rng(1).integers(0, 9, (70, 8))))
    s = Setup([[3, 0]] * 5, 1, 64, page=page, seed=4)
    _run_append(s, 1, 8, flat=True, fused=True, lens_out=lens_out)


def test_append_only_keys_or_queries_are_normalised():
    for name in ("q_norm", "k_norm"):
        _run_append(Setup(LENS, 4, 128, seed=6), 4, 3, **{name: torch.linspace(0.5, 2, 128, device=DEV)})


@pytest.mark.parametrize("page", [0, 16])
def test_append_leaves_pairs_alone(page):
    """No room; a length below zero; rows outside the cache; positions outside the table."""
    s = Setup([[10, 20], [30, 40], [50, 60], [0, 5]], 4, 128, page=page, seed=8)
    s.cap_h = s.cap_h.copy()
    s.cap_h[0, 1] = 23                       # room for three of four
    s.lens_h = s.lens_h.copy()
    s.lens_h[1, 0] = -1
    if page:
        s.pages[5, 3] = s.n_rows // page     # tokens 48 .. 63 of pair 5 in a page that is not there
        s.pages[3, 2] = -1                   # tokens 32 .. 47 of pair 3
    else:
        s.off[5], s.off[3] = s.n_rows - 62, -4
    pos = np.zeros((4, 4), dtype=np.int64)
    pos[2, 1], pos[3, 3] = 9, -1             # of 9 positions
    _run_append(s.make(), 4, 6, table=_table(9, 128, 0), pos=I32(pos))


def test_append_infinities_stay_in_their_rows():
    s = Setup([[4, 4]], 4, 128, "kv8", seed=9)
    q, k, v = _new(s, 3, 4, 0, False)
    k[0, 1, 0, 3], v[0, 1, 1, 5], v[0, 2, 0, 7] = math.inf, -math.inf, math.nan
    before = s.numbers()
    F.fairkv_append_rotated(s.cache, s.lens, q, k, v, torch.empty_like(q), table=_table(4, 64, 0), pos=I32(np.zeros((1, 3))))
    got = s.numbers()
    r = s.row(0, 5)
    assert got[1][s.row(1, 5), 5] == -448 and np.isnan(got[1][s.row(0, 6), 7])
    assert np.abs(got[0][r, 3]) == 448 and np.isfinite(np.delete(got[0][r], [3, 35])).all()
    others = [i for i in range(s.n_rows) if i not in {s.row(p, t) for p in (0, 1) for t in (4, 5, 6)}]
    for a, b in zip(before, got):
        np.testing.assert_array_equal(a[others], b[others])


# ---- accept ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("kv8", 64), ("kv8", 128), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("q_len,page", [(1, 0), (3, 16), (8, 0), (17, 32), (64, 16), (64, 0)])
def test_accept(dtype, D, q_len, page):
    rng = np.random.default_rng(q_len + D)
    B, Hkv = 11, 3
    n_new = rng.integers(0, q_len + 1, B)
    n_new[0] = q_len
    lens = rng.integers(0, 80, (B, Hkv)) + n_new[:, None]
    s = Setup(lens, 0, D, dtype, page, seed=q_len)
    path = np.full((B, q_len), -9)
    n_path = rng.integers(0, n_new + 1)
    n_path[0] = q_len
    for b in range(B):                       # any order, the same row twice
        path[b, :n_path[b]] = rng.integers(0, max(n_new[b], 1), n_path[b]) if b % 2 else np.sort(rng.permutation(n_new[b])[:n_path[b]])
    path[0] = np.arange(q_len)[::-1]
    if q_len > 1:                            # left alone: too many, negative, an entry that is no draft row, a length below the draft's
        n_path[1], n_path[2] = n_new[1] + 1, -1
        n_path[3] = n_new[3] = max(n_new[3], 1)
        path[3, 0] = n_new[3]
        n_new[4] = q_len
        s.lens_h = s.lens_h.copy()
        s.lens_h[4, 1] = q_len - 1
        s.make()
    k0, v0 = s.k.clone(), s.v.clone()
    want, moves, alone = S.accept(s.lens_h, path, n_path, n_new, Hkv, s.row)
    for in_place in (False, True):
        s.k.copy_(k0), s.v.copy_(v0)
        out, bad = torch.full_like(s.lens, -3), torch.zeros(1, dtype=torch.int32, device=DEV)
        F.fairkv_accept(s.cache, s.lens, I32(path), I32(n_path), n_new=I32(n_new), lens_out=None if in_place else out, bad=bad)
        assert (s.lens if in_place else out).cpu().numpy().reshape(-1).tolist() == want.tolist()
        assert int(bad) == len(alone)
        for x, x0 in ((s.k, k0), (s.v, v0)):
            ref = _bits(x0).clone()
            if moves:
                ref[list(moves)] = _bits(x0)[list(moves.values())]
            assert torch.equal(_bits(x), ref)


# ---- attention -------------------------------------------------------------------------------------------
def _workspace(cache, Hq, q_len, n_slots=None):
    """Counters of zero, NaN everywhere else."""
    ws = torch.full((F.fairkv_tree_workspace_bytes(cache, Hq, q_len, n_slots),), 0xff, dtype=torch.uint8, device=DEV)
    F.fairkv_tree_workspace_reset(ws, cache.n_slots if n_slots is None else n_slots)
    return ws


def _attend(s, Hq, q_len, out_dtype, tree=None, n_new=None, n_slots=None, seed=0, scale=None, q=None, stream=None, q_mul=1.0):
    scale = 1 / math.sqrt(s.D) if scale is None else scale
    if q is None:
        q = (torch.randn(s.B, q_len, Hq, s.D, generator=torch.Generator().manual_seed(seed + 1)) * q_mul).to(torch.bfloat16).to(DEV)
    out = torch.full(q.shape, 3.0, dtype=out_dtype, device=DEV)
    lse = torch.full(q.shape[:-1], 3.0, dtype=torch.float32, device=DEV)
    ws = _workspace(s.cache, Hq, q_len, n_slots)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
        ws.record_stream(stream)
    F.fairkv_decode_attn_tree(s.cache, s.lens, q, ws, out, lse, scale, tree=None if tree is None else torch.as_tensor(tree.view(np.int64), device=DEV),
                              n_new=None if n_new is None else I32(n_new), n_slots=n_slots, stream=stream)
    if stream is None:
        counters = ws[:F.fairkv_tree_counter_bytes(s.cache.n_slots if n_slots is None else n_slots)]
        assert not counters.any()            # left as they were found
    return q, out, lse, scale


def _compare(s, q, out, lse, scale, tree, n_new, lens=None):
    B, n, Hq, D = q.shape
    nn = np.full(B, n) if n_new is None else np.clip(n_new, 0, n)
    sees = (lambda b, i, j: j <= i) if tree is None else (lambda b, i, j: bool(int(tree[b, i]) >> j & 1))
    kk, vv = s.numbers()
    heads = np.arange(s.Hkv)
    # scales: of K into q (per head), of V out of the result
    q_h = q.float().cpu().numpy().astype(np.float64).reshape(B, n, s.Hkv, -1, D)
    ref, ref_lse, v_top, s_top = S.attend((q_h * s.ks[heads][None, None, :, None, None]).reshape(B, n, Hq, D), kk, vv, s.lens_h if lens is None else lens, nn, sees, scale, s.Hkv, s.row)
    vs = np.repeat(s.vs, Hq // s.Hkv)[None, None, :, None]
    ref, v_top = ref * vs, v_top * vs[..., 0]
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    live = np.arange(n)[None, :] < nn[:, None]
    assert (got[~live] == 3).all() and (got_lse[~live] == 3).all()
    g, r, gl, rl, vt, st = got[live], ref[live], got_lse[live], ref_lse[live], v_top[live], s_top[live]
    bf16 = out.dtype == torch.bfloat16
    score = st * D * 2.0 ** -24 + 2.0 ** -22
    many = (Hq // s.Hkv) * n > 64
    weight = 2 * score + (2.0 ** -8 if bf16 and many else 2.0 ** -16) + 4096 * 2.0 ** -24
    tol = weight[..., None] * vt[..., None] + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(r)
    seen_inf = ~np.isfinite(r)
    with np.errstate(invalid="ignore"):
        assert np.array_equal(np.isnan(g), np.isnan(r)) and np.array_equal(g[np.isinf(r)], r[np.isinf(r)])
        bad = ~(np.abs(g - r) <= tol) & ~seen_inf
    assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], r[bad][:5])
    none = np.isinf(rl)
    assert (gl[none] == -math.inf).all() and (g[none] == 0).all()
    assert (np.abs(gl[~none] - rl[~none]) <= score[~none] + 4096 * 2.0 ** -24 + 2.0 ** -22 * np.abs(rl[~none])).all()


def _random_tree(B, n, rng, own=True):
    """Ancestors with (or without) the node itself, as bits."""
    bits = np.zeros((B, n), dtype=np.uint64)
    for i in range(n):
        p = rng.integers(-1, i, B) if i else np.full(B, -1)
        bits[:, i] = np.where(p >= 0, bits[np.arange(B), np.maximum(p, 0)] | (np.uint64(1) << np.maximum(p, 0).astype(np.uint64)), 0)
    return bits | (np.uint64(1) << np.arange(n, dtype=np.uint64))[None, :] if own else bits


SHAPES = [(1, 1, 1), (2, 2, 1), (1, 8, 2), (3, 1, 5), (1, 7, 3), (2, 4, 8), (1, 5, 13), (1, 8, 8), (2, 3, 16), (1, 8, 16), (1, 16, 9), (1, 4, 64), (1, 8, 33), (1, 16, 64)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 0), ("bf16", 64, 16), ("kv8", 128, 32), ("kv8", 64, 0)])
@pytest.mark.parametrize("Hkv,G,q_len", SHAPES)
def test_attention_of_a_tree(Hkv, G, q_len, dtype, D, page, out_dtype):
    rng = np.random.default_rng(q_len * 100 + G)
    lens = np.concatenate([[0, 1, 15, 16, 31, 32, 33, 63], rng.integers(40, 400, 4)])
    lens = np.stack([rng.permutation(lens) for _ in range(Hkv)], 1) + q_len
    s = Setup(lens, 1, D, dtype, page, seed=q_len + G, scales=True)
    tree = _random_tree(12, q_len, rng)
    _compare(s, *_attend(s, Hkv * G, q_len, out_dtype, tree), tree, None)


@pytest.mark.parametrize("n_slots", [1, 2, 4, 8, 32])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("bf16", 64, 0), ("kv8", 128, 0), ("kv8", 64, 32)])
@pytest.mark.parametrize("G,q_len", [(4, 13), (8, 16), (8, 24), (4, 64)])
def test_few_workgroups_with_many_columns_each(G, q_len, dtype, D, page, n_slots):
    """The fewer workgroups, the more columns has one: 32 to 256 here."""
    rng = np.random.default_rng(q_len)
    lens = np.array([[400, 33], [0, 129], [31, 257]]) + q_len
    s = Setup(lens, 1, D, dtype, page, seed=q_len + G, scales=True)
    tree = _random_tree(3, q_len, rng)
    n_new = np.array([q_len, q_len - 1, q_len // 2])
    for out_dtype in (torch.float32, torch.bfloat16):
        _compare(s, *_attend(s, 2 * G, q_len, out_dtype, tree, n_new, n_slots, scale=-0.1 if n_slots == 2 else None), tree, n_new)


@pytest.mark.parametrize("n_slots", [2, 5, 9, 24])
@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("kv8", 16)])
@pytest.mark.parametrize("longest", [130, 256, 400])
def test_many_short_pairs_in_a_share(longest, dtype, page, n_slots):
    """Pairs of up to 4 and up to 8 tiles that one wave takes alone, between longer ones and empty ones."""
    rng = np.random.default_rng(longest + n_slots)
    lens = rng.integers(longest // 3, longest + 1, (20, 2))
    lens[3], lens[7, 1], lens[11] = 0, 900, 3
    s = Setup(lens, 0, 128, dtype, page, seed=longest, scales=True)
    n_new = rng.integers(0, 4, 20)
    _compare(s, *_attend(s, 8, 3, torch.float32, None, n_new, n_slots), None, n_new)


@pytest.mark.parametrize("q_len,G", [(1, 4), (4, 8), (16, 4), (40, 8)])
def test_attention_of_a_chain_of_ragged_drafts_and_short_pairs(q_len, G):
    """Pairs without rows, shorter than their draft, drafts of no token, counts out of range: what is no node is left as it was."""
    rng = np.random.default_rng(q_len)
    lens = rng.integers(0, 60, (9, 2))
    lens[0], lens[1, 0] = 0, -3
    n_new = rng.integers(-1, q_len + 3, 9)
    s = Setup(lens, 2, 64, seed=q_len)
    _compare(s, *_attend(s, 2 * G, q_len, torch.float32, None, n_new), None, n_new)


@pytest.mark.parametrize("n_slots", [None, 1, 4])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("G,q_len", [(2, 8), (8, 16), (8, 64)])
def test_masks_that_leave_rows_empty(G, q_len, page, n_slots):
    """Nodes that see nothing at all, nodes that see every draft row, bits behind the draft."""
    rng = np.random.default_rng(5)
    n_new = rng.integers(1, q_len + 1, 6)
    tree = rng.integers(0, 1 << 62, (6, q_len)).astype(np.uint64) << np.uint64(2)
    tree[:, 0], tree[1] = 0, ~np.uint64(0)
    lens = np.stack([n_new, n_new + 40], 1)                # the first head has nothing but the draft
    s = Setup(lens, 0, 128, page=page, seed=1)
    _compare(s, *_attend(s, 2 * G, q_len, torch.float32, tree, n_new, n_slots), tree, n_new)


@pytest.mark.parametrize("n_slots", [None, 1, 2, 8])
@pytest.mark.parametrize("dtype", ["bf16", "kv8"])
@pytest.mark.parametrize("G,q_len", [(4, 6), (8, 12), (8, 40)])
def test_infinite_and_nan_rows_count_for_the_nodes_that_see_them(G, q_len, dtype, n_slots):
    """Values of draft rows that some nodes do not see, rows behind the last one and rows of no pair."""
    rng = np.random.default_rng(11)
    lens = np.array([[50, 33], [q_len, 97]]) + np.array([[q_len], [0]])
    s = Setup(lens, 3, 128, dtype, 16, seed=2)
    tree = _random_tree(2, q_len, rng)
    used = [s.row(p, t) for p in range(4) for t in range(int(lens.reshape(-1)[p]))]
    other = torch.ones(s.n_rows, dtype=torch.bool, device=DEV)
    other[used] = False
    poison = lambda x, at, value: _bits(x).reshape(s.n_rows, -1).__setitem__(at, _bits(torch.full((s.D,), value).to(x.dtype).to(DEV)))
    for x in (s.k, s.v):
        poison(x, other, math.nan)
    values = (math.nan,) if dtype == "kv8" else (math.inf, -math.inf, math.nan)
    for p in range(4):
        for u, value in enumerate(values):
            r = s.row(p, int(lens.reshape(-1)[p]) - 2 - u)
            cell = torch.tensor([value]).to(s.v.dtype).to(DEV)
            _bits(s.v[r])[(u * 7) * s.v.element_size():(u * 7 + 1) * s.v.element_size()] = _bits(cell)
    for out_dtype in (torch.float32, torch.bfloat16):
        _compare(s, *_attend(s, 2 * G, q_len, out_dtype, tree, n_slots=n_slots), tree, None)
    # a NaN key of a row that only some see
    for p in range(4):
        poison(s.k, s.row(p, int(lens.reshape(-1)[p]) - 1), math.nan)
        poison(s.v, s.row(p, int(lens.reshape(-1)[p]) - 1), 1.0)
    q, out, lse, scale = _attend(s, 2 * G, q_len, torch.float32, tree, n_slots=n_slots)
    seen = (tree >> np.uint64(q_len - 1) & np.uint64(1)).astype(bool)
    nan = np.isnan(out.cpu().numpy()).all(-1)
    assert nan[seen].all() and not np.isnan(lse.cpu().numpy())[~seen].any()


@pytest.mark.parametrize("n_slots", [1, 2, 7, 64, 256, 1024, 20000])
@pytest.mark.parametrize("G,q_len", [(1, 1), (8, 5), (8, 12), (4, 64)])
def test_long_pairs_cut_into_many_pieces(G, q_len, n_slots):
    s = Setup([[3000], [70], [9]], 1, 64, page=64, seed=3)
    n_new = np.array([q_len, min(q_len, 60), min(q_len, 9)])
    tree = _random_tree(3, q_len, np.random.default_rng(1))
    _compare(s, *_attend(s, G, q_len, torch.float32, tree, n_new, n_slots), tree, n_new)


def test_more_pairs_than_threads_and_long_tables():
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 40, (171, 4))
    lens[100, 2] = 2000
    s = Setup(lens, 1, 64, page=16, seed=4)
    _compare(s, *_attend(s, 8, 1, torch.float32), None, None)


@pytest.mark.parametrize("q_len", [1, 24])
def test_a_pages_list_longer_than_a_batch_of_64_tiles(q_len):
    """One workgroup alone: 64 tiles of each of its groups of waves are more than one batch of page numbers."""
    s = Setup([[9000 + q_len]], 1, 64, page=16, seed=5)
    _compare(s, *_attend(s, 8, q_len, torch.float32, n_slots=1), None, None)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("kv8", 0)])
def test_one_long_pair_in_more_than_512_pieces(dtype, page):
    """Sums of sums of sums."""
    s = Setup([[20000, 40]], 1, 64, dtype, page, seed=31)
    tree = _random_tree(1, 8, np.random.default_rng(6))
    _compare(s, *_attend(s, 8, 8, torch.float32, tree, n_slots=1500), tree, None)


@pytest.mark.parametrize("expected", [1, 3000, 1 << 40])
def test_a_cache_for_more_rows_than_there_are(expected):
    """However many rows are expected, the results are those of the rows that are there."""
    s = Setup(np.random.default_rng(9).integers(0, 500, (4, 2)), 60000, 64, seed=9)
    where = dict(off=torch.as_tensor(s.off.reshape(4, 2), device=DEV))
    s.cache = F.Cache(s.k, s.v, I32(s.cap_h), expected_rows=expected, **where)
    tree = _random_tree(4, 32, np.random.default_rng(7))
    _compare(s, *_attend(s, 16, 32, torch.float32, tree, n_slots=64), tree, None)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("q_len", [2, 20])
def test_rows_that_the_cache_does_not_have_are_not_attended_to(page, q_len):
    s = Setup([[100, 40], [90, 64]], 1, 128, page=page, seed=6)
    if page:
        s.pages[0, 2], s.pages[1, 0], s.pages[2, 5], s.pages[3, 1] = -1, 1 << 30, s.n_rows // page, -(1 << 31)
    else:
        s.off[0], s.off[3] = s.n_rows - 99, -1
        row = s.row
        s.row = lambda p, t: None if p in (0, 3) else row(p, t)      # a run that does not fit is not read at all
    s.make()
    _compare(s, *_attend(s, 8, q_len, torch.float32), None, None)


def test_lengths_out_of_range():
    """A length beyond the cache is taken as all of it, and a packed run of that many rows does not fit."""
    s = Setup([[20, 30], [40, 9]], 0, 64, page=16, seed=7)
    s.pages[:] = np.arange(s.pages.size).reshape(s.pages.shape) % (s.n_rows // 16)
    s.lens_h = np.array([[2 ** 31 - 1, 30], [-2 ** 31, 9]])
    s.make()
    most = s.pages.shape[1] * 16
    _compare(s, *_attend(s, 8, 1, torch.float32), None, None, lens=np.array([[most, 30], [0, 9]]))
    s = Setup([[20, 30]], 0, 64, seed=7)
    s.lens_h = np.array([[2 ** 31 - 1, 30]])
    s.make()
    _compare(s, *_attend(s, 8, 1, torch.float32), None, None, lens=np.array([[0, 30]]))


def test_scores_that_rise_fall_and_change_sign():
    """The running maximum is raised and the sums are scaled down on the way: ascending scores, large ones, a negative factor, zero."""
    s = Setup([[700, 333]], 1, 128, seed=8)
    direction = torch.randn(128, generator=torch.Generator().manual_seed(1)).to(DEV)
    for p in range(2):
        n = int(s.lens_h[0, p])
        at = [s.row(p, t) for t in range(n)]
        s.k[at] = (direction * torch.linspace(-1.5, 1.5, n, device=DEV)[:, None]).to(torch.bfloat16)
    q = (direction + 0.1 * torch.randn(1, 6, 16, 128, device=DEV)).to(torch.bfloat16)
    for scale in (0.3, -0.3, 0.0, 3.0):
        _compare(s, *_attend(s, 16, 6, torch.float32, q=q, scale=scale), None, None)


def test_one_token_gives_its_value():
    s = Setup([[1, 1]], 1, 128, seed=9)
    for G, q_len in ((1, 1), (16, 1), (8, 8), (8, 16), (8, 40)):
        q, out, lse, _ = _attend(s, 2 * G, q_len, torch.bfloat16, np.full((1, q_len), 1, dtype=np.uint64), np.array([1]))
        for h in range(2):
            assert torch.equal(out[0, 0, h * G:(h + 1) * G], s.v[s.row(h, 0)].expand(G, 128))


def test_the_same_call_gives_the_same_bits():
    s = Setup(np.random.default_rng(0).integers(100, 3000, (4, 2)), 1, 128, seed=10)
    a, b = (_attend(s, 16, 12, torch.float32) for _ in range(2))
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_another_stream_and_no_lse():
    s = Setup([[300, 77]], 1, 128, seed=12)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _attend(s, 8, 3, torch.float32, stream=side)
    side.synchronize()
    _compare(s, *got, None, None)
    q, out = got[0], torch.empty_like(got[1])
    ws = _workspace(s.cache, 8, 3)
    F.fairkv_decode_attn_tree(s.cache, s.lens, q, ws, out, None, got[3])
    assert torch.equal(out, got[1])


def test_calls_refuse_what_does_not_fit_the_cache():
    s = Setup([[30, 7]], 4, 128, seed=13)
    q, k, v = _new(s, 2, 4, 0, False)
    n = lambda *d: torch.zeros(d, dtype=torch.int32, device=DEV)
    out, ws = torch.empty_like(q), torch.empty(F.fairkv_tree_workspace_bytes(s.cache, 4, 2), dtype=torch.uint8, device=DEV)
    good = dict(lens=s.lens, q=q, k_new=k, v_new=v, q_out=out)
    for change in (dict(lens=n(3)), dict(q=q[..., :64]), dict(k_new=k[:, :1]), dict(v_new=v[:, :, :1]), dict(q_out=out[:, :1]), dict(q=q[0]), dict(lens=s.lens.long()),
                   dict(q=torch.empty(1, 4, 2, 128, dtype=q.dtype, device=DEV).transpose(1, 2)), dict(n_new=n(2)), dict(lens_out=n(1)), dict(bad=n(2)),
                   dict(table=_table(4, 64, 0)), dict(table=_table(4, 64, 0), pos=n(1, 1)), dict(q_norm=torch.ones(64, device=DEV)), dict(lens=s.lens.cpu())):
        with pytest.raises(ValueError):
            F.fairkv_append_rotated(s.cache, **{**good, **change})
    with pytest.raises(TypeError):
        F.fairkv_append_rotated(s.cache, **{**good, "q": q.float()})
    with pytest.raises(F.FairKVError):
        F.fairkv_append_rotated(s.cache, **good, table=_table(4, 24, 0), pos=n(1, 2))
    good = dict(lens=s.lens, q=q, workspace=ws, out=out, lse=None, scale=1.0)
    for change in (dict(lens=n(1)), dict(out=out[..., :64]), dict(tree=n(1, 2)), dict(tree=torch.zeros(1, 3, dtype=torch.int64, device=DEV)), dict(lse=torch.empty(1, 2, 3, device=DEV)),
                   dict(n_new=n(2)), dict(q=q.transpose(1, 2))):
        with pytest.raises(ValueError):
            F.fairkv_decode_attn_tree(s.cache, **{**good, **change})
    with pytest.raises(F.FairKVError):
        F.fairkv_decode_attn_tree(s.cache, **{**good, "workspace": ws[:-16]})
    for change in (dict(path=n(2)), dict(path=n(2, 2)), dict(n_path=n(2)), dict(lens=n(1)), dict(path=n(1, 2).long())):
        with pytest.raises(ValueError):
            F.fairkv_accept(s.cache, **{**dict(lens=s.lens, path=n(1, 2), n_path=n(1)), **change})


# ---- a step ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("bf16", 16), ("kv8", 32)])
def test_steps_captured_once_and_replayed_while_the_cache_grows(dtype, page):
    """append, attend, accept, over and over: one graph, the lengths and the page lists read on the GPU; every replay against the oracle, and
    two graphs that share a workspace in turn."""
    B, Hkv, G, q_len, D, steps = 3, 2, 4, 6, 128, 4
    rng = np.random.default_rng(2)
    s = Setup(rng.integers(0, 60, (B, Hkv)), steps * q_len, D, dtype, page, seed=20, scales=True)
    Hq = Hkv * G
    q, k_new, v_new = (x.clone() for x in _new(s, q_len, Hq, 0, False))
    kw = dict(table=_table(64, D, 1), pos=I32(np.zeros((B, q_len))), q_norm=torch.ones(D, device=DEV), k_norm=torch.ones(D, device=DEV), pairs=True)
    tree = torch.zeros(B, q_len, dtype=torch.int64, device=DEV)
    n_new, path, n_path = I32(np.zeros(B)), I32(np.zeros((B, q_len))), I32(np.zeros(B))
    q_out, bad = torch.zeros_like(q), I32([0])
    ws = _workspace(s.cache, Hq, q_len)
    outs = [(torch.zeros(q.shape, device=DEV), torch.zeros(q.shape[:-1], device=DEV)) for _ in range(2)]
    grown = torch.zeros_like(s.lens)

    def step(out, lse):
        F.fairkv_append_rotated(s.cache, s.lens, q, k_new, v_new, q_out, n_new=n_new, lens_out=grown, bad=bad, **kw)
        F.fairkv_decode_attn_tree(s.cache, grown, q_out, ws, out, lse, 0.1, tree=tree, n_new=n_new)
        F.fairkv_accept(s.cache, grown, path, n_path, n_new=n_new, lens_out=s.lens, bad=bad)

    graphs = []
    for out, lse in outs:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(out, lse)                   # n_new is 0: nothing happens
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(out, lse)
        graphs.append(g)
    for i in range(steps):
        nn = rng.integers(1, q_len + 1, B)
        bits = _random_tree(B, q_len, rng)
        kept = rng.integers(0, nn + 1)
        chosen = np.full((B, q_len), -1)
        for b in range(B):
            chosen[b, :kept[b]] = np.sort(rng.permutation(nn[b])[:kept[b]])
        for t, x in ((n_new, nn), (path, chosen), (n_path, kept), (kw["pos"], rng.integers(0, 64, (B, q_len)))):
            t.copy_(I32(x))
        tree.copy_(torch.as_tensor(bits.view(np.int64), device=DEV))
        for t in (q, k_new, v_new):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(i)).to(t.dtype))
        before, q_before, lens_before = (s.k.clone(), s.v.clone()), q_out.clone(), s.lens.cpu().numpy().astype(np.int64)
        out, lse = outs[i % 2]
        out.fill_(3.0), lse.fill_(3.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        after = (s.k.clone(), s.v.clone())
        # what the accept moved, taken back: the cache as the attention saw it
        s.lens_h = lens_before
        _, moves, alone = S.accept(grown.cpu().numpy(), chosen, kept, nn, Hkv, s.row)
        assert not alone and int(bad) == 0
        F.fairkv_append_rotated(s.cache, I32(lens_before), q, k_new, v_new, torch.empty_like(q), n_new=n_new, lens_out=torch.empty_like(s.lens), **kw)
        _check_append(s, q, k_new, v_new, q_out, before, q_before, grown, None, kw, nn)
        s.lens_h = grown.cpu().numpy().astype(np.int64)
        _compare(s, q_out, out, lse, 0.1, bits, nn)
        for x, y in zip((s.k, s.v), after):
            ref = _bits(x).clone()
            if moves:
                ref[list(moves)] = _bits(x)[list(moves.values())]
            assert torch.equal(ref, _bits(y))
            x.copy_(y)
        assert s.lens.cpu().numpy().tolist() == (lens_before + kept[:, None]).tolist()


@pytest.mark.parametrize("page", [0, 64])
def test_rows_behind_4_gib_are_those_that_are_meant(page):
    """The same steps near the front of a cache and behind byte 2^32 of it: the same bits."""
    B, Hkv, G, q_len, D, each = 2, 2, 4, 5, 128, 320
    n_rows = (1 << 24) + 4096
    k, v = (torch.empty(n_rows, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens = np.array([[200, 31], [300, 0]])
    firsts = (64, (1 << 24) + 64)            # of B * Hkv runs of `each` rows
    old = [torch.randn(B * Hkv * each, D, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(DEV) for i in range(2)]
    q, k_new, v_new = (torch.randn(B, q_len, h, D, generator=torch.Generator().manual_seed(h)).to(torch.bfloat16).to(DEV) for h in (Hkv * G, Hkv, Hkv))
    path, n_path = I32([[4, 1, 2, 0, 0], [3, 4, 0, 0, 0]]), I32([3, 2])
    results = []
    for first in firsts:
        at = slice(first, first + B * Hkv * each)
        k[at], v[at] = old[0], old[1]
        where = dict(off=torch.arange(B * Hkv, device=DEV).view(B, Hkv) * each + first) if not page else \
            dict(pages=I32((first + np.arange(B * Hkv * each).reshape(B * Hkv, -1)[:, ::page]) // page), page_rows=page)
        cache = F.Cache(k, v, I32(np.full((B, Hkv), each)), **where)
        t, q_out, out, lse = I32(lens), torch.empty_like(q), torch.empty(q.shape, device=DEV), torch.empty(q.shape[:-1], device=DEV)
        F.fairkv_append_rotated(cache, t, q, k_new, v_new, q_out, q_norm=torch.ones(D, device=DEV))
        F.fairkv_decode_attn_tree(cache, t, q_out, _workspace(cache, Hkv * G, q_len), out, lse, 0.1)
        F.fairkv_accept(cache, t, path, n_path)
        results.append((t, q_out, out, lse, k[at].clone(), v[at].clone()))
    assert not torch.equal(results[0][4], old[0])
    for near, far in zip(*results):
        assert torch.equal(near, far)


@pytest.mark.parametrize("Hq,Hkv,D,B,q_len", [(80, 1, 128, 48, 64), (5, 1, 128, 160, 64), (1, 1, 64, 1100, 64), (16, 2, 128, 3000, 1)])
def test_many_tokens_in_a_workgroup_give_what_few_give(Hq, Hkv, D, B, q_len):
    """So many tokens that workgroups of the queries make several passes, against calls of a few sequences each."""
    rng = np.random.default_rng(Hq)
    n_new = rng.integers(0, q_len + 1, B)
    n_new[B // 2: B // 2 + 3] = 0
    lens = rng.integers(0, 9, (B, Hkv))
    s = Setup(lens, q_len, D, seed=Hq)
    q, k_new, v_new = _new(s, q_len, Hq, 1, True)
    pos = rng.integers(0, 32, (B, q_len))
    pos[rng.integers(0, B, 20), rng.integers(0, q_len, 20)] = 32      # outside the table
    kw = dict(table=_table(32, 32, 0), q_norm=torch.rand(D, device=DEV), k_norm=torch.rand(D, device=DEV))
    k0, v0 = s.k.clone(), s.v.clone()

    def run(per_call):
        s.k.copy_(k0), s.v.copy_(v0)
        q_out, bad, grown = torch.full((B, q_len, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV), I32([0]), I32(np.full((B, Hkv), -1))
        for b in range(0, B, per_call):
            at = slice(b, min(b + per_call, B))
            cache = F.Cache(s.k, s.v, I32(s.cap_h[at]), off=torch.as_tensor(s.off.reshape(B, Hkv)[at].copy(), device=DEV))
            F.fairkv_append_rotated(cache, I32(lens[at]), q[at], k_new[at], v_new[at], q_out[at], pos=I32(pos[at]), n_new=I32(n_new[at]),
                                    lens_out=grown[at], bad=bad, **kw)
        return q_out, bad, grown, s.k.clone(), s.v.clone()

    for many, few in zip(run(B), run(16 if q_len > 1 else 500)):
        assert torch.equal(many, few)


def test_two_streams_at_once_with_a_workspace_each():
    s = Setup(np.random.default_rng(3).integers(0, 900, (6, 4)), 0, 128, seed=21)
    q, out, lse, scale = _attend(s, 32, 12, torch.float32)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [_workspace(s.cache, 32, 12) for _ in streams]
    got = [[(torch.empty_like(out), torch.empty_like(lse)) for _ in range(4)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(4):
        for stream, ws, results in zip(streams, spaces, got):
            F.fairkv_decode_attn_tree(s.cache, s.lens, q, ws, *results[i], scale, stream=stream)
    torch.cuda.synchronize()
    for x in got[0] + got[1]:
        assert torch.equal(x[0], out) and torch.equal(x[1], lse)
