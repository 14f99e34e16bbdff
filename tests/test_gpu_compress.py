"""Compression of a growing cache on the GPU against the oracle: attention weights added up, selection, eviction, and the three behind a step.

Tolerance of a weight w = exp(z - lse) (fp32 numbers are off by at most 2^-24 of themselves), relative to w:
  scores    D products summed in fp32: at most D 2^-24 of S = scale sum_d |q_d k_d|; the factor to log2 units is the product of three numbers, each rounded
            (3 2^-24 |z|), the log-sum-exp is one product (2^-24 |lse|), their difference is rounded once (2^-24 (|z| + |lse|)); a log2 unit is ln 2 of
            these.  The exponential itself: one unit in the last place, 2^-23.
  sums      of n weights and one old one, all positive: n 2^-24 of the sum, a product and a sum with the old one, 2 2^-24.
Selections and moves are exact."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import compress as C
from oracle import step as S
from test_gpu_step import DEV, I32, TYPES, Setup, _bits

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _fits(s):
    if s.page:
        return None
    return lambda p: s.off[p] >= 0 and s.off[p] + max(int(s.lens_h.reshape(-1)[p]), 0) <= s.n_rows


def _words(B, n, seed):
    rng = np.random.default_rng(seed)
    bits = np.zeros((B, n), dtype=np.uint64)
    for b in range(B):
        for i in range(n):
            up = int(rng.integers(-1, i)) if i else -1
            bits[b, i] = (bits[b, up] if up >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(i))
    return bits


def _lse(s, q, scale, n_new, tree):
    """Of all scores that a node sees; a node behind the sequence's last has a NaN there, which must not be read."""
    k, _ = s.numbers()
    B, n, Hq, _ = q.shape
    G = Hq // s.Hkv
    out = np.full((B, n, Hq), np.nan)
    for b in range(B):
        for h in range(s.Hkv):
            length, m = int(s.lens_h[b, h]), int(n_new[b])
            at = [s.row(b * s.Hkv + h, t) for t in range(length)]
            t = np.array([x for x in range(length) if at[x] is not None], dtype=np.int64)
            kk = k[[at[x] for x in t]] * s.ks[h]
            for i in range(m):
                word = (1 << (i + 1)) - 1 if tree is None else int(tree[b, i])
                sees = np.array([x < length - m or word >> int(x - length + m) & 1 for x in t], dtype=bool)
                for g in range(h * G, (h + 1) * G):
                    z = scale * (kk[sees] @ q[b, i, g]) if sees.any() else np.zeros(0)
                    top = z.max() if z.size else -np.inf
                    out[b, i, g] = top + math.log(np.exp(z - top).sum()) if np.isfinite(top) else top
    return out


def _weight_tolerance(s, q, lse, scale, n_new, tree, old, decay, want):
    """Per row, as the file's head has it."""
    k, _ = s.numbers()
    B, n, Hq, D = q.shape
    G = Hq // s.Hkv
    tol = np.zeros(s.n_rows)
    for b in range(B):
        for h in range(s.Hkv):
            rows = [r for r in (s.row(b * s.Hkv + h, t) for t in range(int(s.lens_h[b, h]))) if r is not None]
            kk = k[rows] * s.ks[h]
            for i in range(int(n_new[b])):
                for g in range(h * G, (h + 1) * G):
                    if not np.isfinite(lse[b, i, g]):
                        continue
                    z, big = scale * (kk @ q[b, i, g]), abs(scale) * (np.abs(kk) @ np.abs(q[b, i, g]))
                    rel = D * big + 4 * np.abs(z) + 2 * abs(lse[b, i, g]) + 2
                    tol[rows] += np.exp(np.minimum(z - lse[b, i, g], 1.0)) * rel * U      # unseen rows too: more than their share
    return tol * 1.01 + U * (int(np.max(n_new)) * G + 3) * np.abs(want) + 2 * U * np.abs(decay * old) + 1e-37


CASES = [
    # dtype, D, Hkv, G, q_len, lens, page, tree, ragged, decay
    ("bf16", 128, 2, 8, 1, [[5, 130], [1, 33]], 0, False, False, 1.0),
    ("bf16", 128, 1, 1, 1, [[1], [31], [32], [129]], 16, False, False, 0.0),
    ("bf16", 64, 3, 5, 7, [[7, 64, 200], [9, 7, 31]], 16, True, True, 0.5),
    ("bf16", 128, 2, 16, 64, [[64, 300], [150, 65]], 32, True, False, 1.0),
    ("bf16", 64, 2, 16, 3, [[600, 3], [257, 255]], 0, False, True, -0.5),
    ("kv8", 128, 2, 8, 2, [[40, 500], [2, 90]], 16, False, False, 0.9),
    ("kv8", 64, 4, 3, 9, [[9, 10, 11, 300], [127, 128, 129, 33]], 0, True, True, 0.0),
    ("kv8", 128, 1, 7, 64, [[70], [641]], 64, False, True, 1.0),
    ("bf16", 128, 2, 4, 5, [[0, 3], [1, 5], [4, 0]], 0, False, False, 1.0),            # shorter than the draft, none at all
    ("bf16", 64, 1, 2, 2, [[n] for n in range(1, 70, 3)], 16, True, False, 0.25),
    ("bf16", 128, 8, 8, 1, [[1200, 5, 90, 17, 2500, 3, 64, 128]], 16, False, False, 1.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-D{c[1]}-{c[2]}x{c[3]}-q{c[4]}-p{c[6]}")
def test_weights(case):
    dtype, D, Hkv, G, n, lens, page, tree, ragged, decay = case
    s = Setup(lens, 5, D, dtype, page, seed=n, scales=True)
    rng = np.random.default_rng(n + D)
    B, Hq, scale = s.B, Hkv * G, 1.0 / math.sqrt(D)
    n_new = rng.integers(0, n + 1, B) if ragged else np.full(B, n)
    words = _words(B, n, n) if tree else None
    q = torch.randn(B, n, Hq, D, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16)
    q_h = q.double().numpy()
    lse = _lse(s, q_h, scale, n_new, words).astype(np.float32)
    old = np.exp(rng.standard_normal(s.n_rows)).astype(np.float32)
    if not decay:
        old[:] = np.nan                              # is not read
    want = C.attn_weights(q_h, s.numbers()[0], s.lens_h, lse, old, scale, decay, n_new, words, s.row, s.ks, _fits(s))
    tol = _weight_tolerance(s, q_h, lse.astype(np.float64), scale, n_new, words, np.nan_to_num(old), decay, np.nan_to_num(want))
    kw = dict(tree=None if words is None else torch.from_numpy(words.view(np.int64)).to(DEV), n_new=I32(n_new) if ragged else None, decay=decay)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    q, lse, first = q.to(DEV), dev(lse), dev(old)
    other = dev(old)
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, first, scale, weights_out=other, **kw)
    assert torch.equal(first.nan_to_num(), dev(old).nan_to_num())
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, first, scale, n_slots=7, **kw)
    assert torch.equal(first.nan_to_num(), other.nan_to_num())      # in place, and by other shares: the same sums
    got = other.double().cpu().numpy()
    assert (np.isnan(got) == np.isnan(want)).all()
    off = np.abs(np.nan_to_num(got) - np.nan_to_num(want))
    assert (off <= tol).all(), (np.max(off / tol), np.argmax(off / tol))
    touched = {r for p in range(B * Hkv) for t in range(int(s.lens_h.reshape(-1)[p])) if (r := s.row(p, t)) is not None}
    rest = np.array(sorted(set(range(s.n_rows)) - touched))
    assert np.array_equal(got[rest], old[rest].astype(np.float64), equal_nan=True)


@pytest.mark.parametrize("D,G,n,ragged", [(128, 8, 9, False), (128, 5, 40, True), (128, 8, 33, True), (64, 16, 64, True), (128, 16, 64, False), (64, 8, 16, False), (128, 16, 40, True),
                                          (128, 16, 33, False)])
def test_weights_are_the_same_whoever_computes_them(D, G, n, ragged):
    """A sequence by itself and beside others, over few workgroups and many: tiles that one wave has or several, all bits the same."""
    lens = np.array([[n + 1, 700], [33 + n, 290], [64, 1500]])
    s = Setup(lens, 5, D, page=16, seed=n)
    gen = torch.Generator().manual_seed(n)
    q = torch.randn(3, n, 2 * G, D, generator=gen).to(torch.bfloat16).to(DEV)
    lse = (3 + torch.rand(3, n, 2 * G, generator=gen)).to(DEV)
    n_new = I32([n, n // 2, n - 1]) if ragged else None
    want = None
    for n_slots in (1, 2, 13, 256, 1000):
        out = torch.full((s.n_rows,), 0.5, device=DEV)
        F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, n_new=n_new, n_slots=n_slots)
        want = out if want is None else want
        assert torch.equal(out, want)
    out = torch.full((s.n_rows,), 0.5, device=DEV)
    for b in range(3):
        alone = torch.zeros_like(s.lens)
        alone[b] = s.lens[b]
        F.fairkv_attn_weights(s.cache, alone, q, lse, out, 0.1, n_new=n_new)
    assert torch.equal(out, want)


def test_rows_that_are_no_numbers_count_where_they_are_seen():
    s = Setup([[70, 40]], 2, 128, page=16)
    n, Hq = 4, 4
    q = torch.randn(1, n, Hq, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    words = np.array([[0b0001, 0b0011, 0b0101, 0b1101]], dtype=np.uint64)      # node 1 is seen by itself only
    lse = torch.from_numpy(_lse(s, q.double().cpu().numpy(), 0.1, [n], words).astype(np.float32)).to(DEV)
    kw = dict(tree=torch.from_numpy(words.view(np.int64)).to(DEV))
    out = torch.zeros(s.n_rows, device=DEV)
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, **kw)
    row = s.row(0, 70 - n + 1)
    s.k[row] = math.inf
    lse[:, 1] = -math.inf                            # node 1 gives nothing: nobody is left who sees that row
    want = out.clone()
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, **kw)
    assert float(out[row]) == 0.0 or math.isnan(float(out[row]))
    s.k[row] = math.nan
    words[0, 1] = 0b0001
    kw["tree"] = torch.from_numpy(words.view(np.int64)).to(DEV)
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, **kw)
    assert float(out[row]) == 0.0
    assert bool(torch.isfinite(out).all())
    others = [s.row(0, t) for t in range(66) if t]
    assert bool((out[others] <= want[others]).all())


def test_log_sum_exps_that_are_no_numbers():
    s = Setup([[40]], 0, 64)
    q = torch.randn(1, 2, 2, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    rows = [s.row(0, t) for t in range(40)]
    out, other = torch.zeros(s.n_rows, device=DEV), torch.zeros(s.n_rows, device=DEV)
    base = torch.tensor([[[2.0, 3.0], [2.5, 1.0]]], device=DEV)
    for value in (math.inf, -math.inf):              # either way this node gives nothing
        lse = base.clone()
        lse[0, 0] = value
        F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1)
        F.fairkv_attn_weights(s.cache, s.lens, q[:, 1:].contiguous(), base[:, 1:].contiguous(), other, 0.1)
        assert torch.equal(out[rows], other[rows])
    lse = base.clone()
    lse[0, 0, 0] = math.nan
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1)
    assert bool(torch.isnan(out[rows[:-1]]).all()) and bool(torch.isfinite(out[rows[-1]]))      # the last row is the other node's own


def test_a_packed_run_that_sticks_out_and_pages_that_are_none():
    s = Setup([[40, 50], [30, 20]], 0, 64)
    s.off[1] = s.n_rows - 20
    s.off[2] = -3
    s.make()
    q = torch.randn(2, 2, 64, device=DEV).to(torch.bfloat16)
    lse = torch.zeros(2, 2, device=DEV)
    out = torch.full((s.n_rows,), 7.0, device=DEV)
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, decay=0.0)
    touched = set(range(int(s.off[0]), int(s.off[0]) + 40)) | set(range(int(s.off[3]), int(s.off[3]) + 20))
    changed = set(torch.nonzero(out != 7.0).flatten().tolist())
    assert changed == touched
    p = Setup([[100]], 0, 64, page=16)
    p.pages[0, 2], p.pages[0, 4] = -1, p.n_rows // 16
    p.make()
    out = torch.full((p.n_rows,), 7.0, device=DEV)
    F.fairkv_attn_weights(p.cache, p.lens, q[:1, :1], lse[:1, :1].contiguous(), out, 0.1)
    want = {p.row(0, t) for t in range(100)} - {None}
    assert len(want) == 68 and set(torch.nonzero(out != 7.0).flatten().tolist()) == want


def test_lengths_and_counts_beyond_their_range():
    s = Setup([[20], [20]], 0, 64, page=16)
    q = torch.randn(2, 3, 2, 64, device=DEV).to(torch.bfloat16)
    lse = torch.zeros(2, 3, 2, device=DEV)
    out = torch.zeros(s.n_rows, device=DEV)
    F.fairkv_attn_weights(s.cache, I32([[-5], [1 << 30]]), q, lse, out, 0.1, n_new=I32([9, -2]))
    seen = torch.nonzero(out).flatten().tolist()
    assert not seen                                  # no rows; no queries
    F.fairkv_attn_weights(s.cache, I32([[-2 ** 31], [2 ** 31 - 1]]), q, lse, out, 0.1, n_new=I32([2 ** 31 - 1, 1]))
    assert not torch.nonzero(out[[s.row(0, t) for t in range(20)]]).numel()


# ---- select ------------------------------------------------------------------------------------------------
def _check_select(s, w, budget, shared, pool=1, sink=0, recent=0, max_keep=None, n_slots=None):
    lens = np.maximum(s.lens_h, 0)
    most = int(lens.max()) + 2 if max_keep is None else max_keep
    lists, counts = C.select(w.astype(np.float64), s.lens_h, budget, shared, pool, sink, recent, most, s.row)
    keep = torch.full((s.B, s.Hkv, most), -9, dtype=torch.int32, device=DEV)
    n_keep, bad = torch.full((s.B, s.Hkv), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.zeros(F.fairkv_select_workspace_bytes(s.cache, shared, n_slots), dtype=torch.uint8, device=DEV)
    for call in range(2):                            # what has to be zero is left so
        F.fairkv_select(s.cache, s.lens, torch.from_numpy(w).to(DEV), I32(budget), keep, n_keep, ws, pool=pool, sink=sink, recent=recent, bad=bad, n_slots=n_slots)
        assert n_keep.cpu().numpy().tolist() == counts.tolist()
        got = keep.cpu().numpy().reshape(-1, most)
        for p, want in enumerate(lists):
            if len(want) <= most:
                assert got[p, :len(want)].tolist() == want, p
                assert (got[p, len(want):] == -9).all()
        assert int(bad) == (call + 1) * int((counts < 0).sum())
    assert not int(ws[:ws.numel() // 3].max())
    return lists


def _some_weights(n, seed, kind):
    rng = np.random.default_rng(seed)
    if kind == "tail":
        w = np.exp(2 * rng.standard_normal(n))
        w[rng.random(n) < 0.1] = 0
    elif kind == "few":                              # many ties
        w = rng.integers(0, 3, n).astype(np.float64)
    elif kind == "equal":
        w = np.full(n, 0.125)
    elif kind == "near":                             # neighbours among the floats
        w = (np.float32(1.0).view(np.int32) + rng.integers(0, 5, n)).astype(np.int32).view(np.float32)
    else:                                            # signs, zeros of both, no numbers
        w = rng.choice([-2.0, -0.0, 0.0, 1.0, math.inf, -math.inf, math.nan, 1e-40, -1e-40, 3.0], n)
    return np.ascontiguousarray(w, dtype=np.float32)


LENS = {"mixed": [[0, 5, 300], [1, 1500, 64], [33, 2, 1030]], "one": [[1]], "long": [[5000, 40], [3, 9000]], "even": [[64] * 8] * 5}


@pytest.mark.parametrize("kind", ["tail", "few", "equal", "near", "signs"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("lens,page", [("mixed", 0), ("mixed", 16), ("long", 32), ("one", 0), ("even", 16)])
def test_selection(lens, page, shared, kind):
    s = Setup(LENS[lens], 1, 64, page=page)
    w = _some_weights(s.n_rows, 3, kind)
    total = np.maximum(s.lens_h, 0).sum(1) if shared else s.lens_h
    for part, pool, sink, recent in ((0.5, 1, 0, 0), (0.1, 5, 4, 32), (0.9, 3, 1, 0), (0.3, 63, 0, 7)):
        _check_select(s, w, np.rint(total * part), shared, pool, sink, recent)


@pytest.mark.parametrize("shared", [False, True])
def test_budgets_at_their_ends(shared):
    s = Setup([[40, 7, 0], [100, 1, 3]], 0, 64, page=16)
    w = _some_weights(s.n_rows, 1, "tail")
    groups = 2 if shared else 6
    for budget in (0, -5, -2 ** 31, 1, 2 ** 31 - 1, 41, 39):
        _check_select(s, w, np.full(groups, budget), shared, 3, 2, 3)
    _check_select(s, w, np.full(groups, 50), shared, 1, 2 ** 31 - 1, 0)
    _check_select(s, w, np.full(groups, 50), shared, 1, 0, 2 ** 31 - 1)
    _check_select(s, w, np.full(groups, 50), shared, 1, 2 ** 31 - 1, 2 ** 31 - 1)


def test_more_than_there_is_room_for_is_counted():
    s = Setup([[40, 7, 90], [100, 1, 3]], 0, 64)
    w = _some_weights(s.n_rows, 2, "tail")
    _check_select(s, w, [60, 60], True, max_keep=20)
    _check_select(s, w, [[5, 7, 21], [20, 9, 9]], False, max_keep=20)


def test_selection_over_rows_that_are_not_there():
    s = Setup([[100, 40]], 0, 64, page=16)
    s.pages[0, 1], s.pages[0, 3], s.pages[1, 2] = -1, s.n_rows, -1
    s.make()
    w = _some_weights(s.n_rows, 2, "tail")
    for budget, sink, recent in (([50], 0, 0), ([90], 20, 60), ([200], 4, 4)):
        _check_select(s, w, budget, True, 5, sink, recent)
    s = Setup([[40, 50], [30, 20]], 0, 64)
    s.off[1], s.off[2] = s.n_rows - 20, -3
    s.make()
    w = _some_weights(s.n_rows, 2, "tail")
    _check_select(s, w, [45, 30], True, 3, 2, 8)
    s.lens_h[:] = [[-4, 2], [3, -1]]
    s.make()
    _check_select(s, w, [45, 30], True, 3, 2, 8)


@pytest.mark.parametrize("kind", ["tail", "near", "equal"])
@pytest.mark.parametrize("lens,shared,n_slots", [([[70000, 40000]], True, None), ([[30000], [200]], False, None), ([[9000] * 8], True, 3), ([[20000, 1], [1, 20000]], True, None)])
def test_long_pairs(lens, shared, n_slots, kind):
    s = Setup(lens, 0, 64, page=64)
    w = _some_weights(s.n_rows, 5, kind)
    total = s.lens_h.sum(1) if shared else s.lens_h
    _check_select(s, w, np.rint(total * 0.06), shared, 5, 4, 32, n_slots=n_slots)
    _check_select(s, w, np.rint(total * 0.8), shared, 1, 0, 64, n_slots=n_slots)


@pytest.mark.parametrize("pool", [1, 3])
def test_groups_of_as_many_rows_as_a_workgroup_has_and_of_more(pool):
    s = Setup([[7616], [7680], [7681], [10239], [10240], [10241], [12289], [30000], [1]], 0, 64, page=64)
    w = _some_weights(s.n_rows, 6, "near")
    for part in (0.03, 0.7):
        _check_select(s, w, np.rint(s.lens_h * part), False, pool, 2, 16)
    pairs = Setup([[5000, 5240], [5001, 5240], [1, 7680], [40, 7700]], 0, 64, page=64, seed=1)
    _check_select(pairs, _some_weights(pairs.n_rows, 7, "near"), np.rint(pairs.lens_h.sum(1) * 0.4), True, pool, 2, 16)


@pytest.mark.parametrize("last", [0, 1, 511, 1022, 1023])
def test_weights_that_differ_in_their_last_bits(last):
    """All in one bin of the first two digits; the budget ends at ties, in front of them and behind them."""
    s = Setup([[9000, 13000], [30, 200]], 0, 64, page=64)
    rng = np.random.default_rng(last)
    bits = rng.integers(0, 1024, s.n_rows)
    bits[rng.random(s.n_rows) < 0.3] = last          # ties
    w = (np.float32(1.0).view(np.uint32) + bits.astype(np.uint32)).view(np.float32)
    at = np.array([s.row(p, t) for p in (0, 1) for t in range(int(s.lens_h[0, p]))])
    above, ties = int((bits[at] > last).sum()), int((bits[at] == last).sum())
    for budget in (above + 1, above + ties // 2, above + ties, above + ties + 1, max(above, 1)):
        _check_select(s, w, np.array([budget, 50]), True)
    _check_select(s, w, np.rint(s.lens_h * 0.5), False)


@pytest.mark.parametrize("shared", [False, True])
def test_more_heads_than_a_workgroup_keeps_in_mind(shared):
    rng = np.random.default_rng(2)
    s = Setup(rng.integers(0, 90, (3, 80)), 0, 64, page=16)
    s.lens_h[1] = 0                                  # a sequence without rows
    s.make()
    w = _some_weights(s.n_rows, 4, "tail")
    total = s.lens_h.sum(1) if shared else s.lens_h
    for part, pool, sink, recent in ((0.4, 3, 2, 8), (0.0, 1, 0, 0), (2.0, 1, 0, 0)):
        _check_select(s, w, np.rint(total * part), shared, pool, sink, recent)


def test_pairs_that_share_rows_are_refused_not_followed_out_of_the_workspace():
    """Rows of different pairs must not overlap; where they do, a group may have more rows than the workspace was made for."""
    for n_pages in (40, 400):                        # no group can be a large one; one can, and has fewer blocks
        s = Setup([[n_pages * 64]], 0, 64, page=64)
        pages = np.arange(n_pages, dtype=np.int32)[None, None].repeat(64, 1)
        lens = I32(np.full((1, 64), n_pages * 64))
        cache = F.Cache(s.k, s.v, lens, pages=I32(pages), page_rows=64)
        keep, n_keep = torch.zeros(1, 64, 8, dtype=torch.int32, device=DEV), torch.zeros(1, 64, dtype=torch.int32, device=DEV)
        ws, bad = torch.zeros(F.fairkv_select_workspace_bytes(cache, True), dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        guard = torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV)
        F.fairkv_select(cache, lens, torch.ones(s.n_rows, device=DEV), I32([100]), keep, n_keep, ws, bad=bad)
        assert (n_keep == -1).all() and int(bad) == 64 and bool((guard == 7).all())


def test_one_workspace_for_calls_of_all_shapes():
    a, b, c = Setup([[9000, 12000]], 0, 64, page=64), Setup([[300] * 8] * 3, 0, 64), Setup([[40000], [20000], [3]], 0, 64)
    need = max(F.fairkv_select_workspace_bytes(x.cache, sh) for x in (a, b, c) for sh in (False, True))
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    F.fairkv_select_workspace_reset(ws)
    for turn in range(3):
        for s in (a, c, b):
            for shared in (turn % 2 == 0, turn % 2 == 1):
                w = _some_weights(s.n_rows, turn, "tail")
                budget = np.rint((s.lens_h.sum(1) if shared else s.lens_h) * 0.3)
                most = int(s.lens_h.max())
                lists, counts = C.select(w.astype(np.float64), s.lens_h, budget, shared, 1, 0, 4, most, s.row)
                keep, n_keep = torch.zeros(s.B, s.Hkv, most, dtype=torch.int32, device=DEV), torch.zeros(s.B, s.Hkv, dtype=torch.int32, device=DEV)
                F.fairkv_select(s.cache, s.lens, torch.from_numpy(w).to(DEV), I32(budget), keep, n_keep, ws, recent=4)
                assert n_keep.cpu().numpy().tolist() == counts.tolist()
                got = keep.cpu().numpy().reshape(-1, most)
                assert all(got[p, :len(x)].tolist() == x for p, x in enumerate(lists))


# ---- evict -------------------------------------------------------------------------------------------------
def _lists(lens, part, seed):
    rng = np.random.default_rng(seed)
    most = max(1, int(lens.max()))
    keep, counts = np.full(lens.shape + (most,), -3, dtype=np.int32), np.zeros(lens.shape, dtype=np.int32)
    for at in np.ndindex(*lens.shape):
        n = int(rng.binomial(lens[at], part))
        keep[at][:n], counts[at] = np.sort(rng.permutation(lens[at])[:n]), n
    return keep, counts


def _moved(x, moves, into=None):
    out = x.clone() if into is None else into.clone()
    if moves:
        to, frm = (torch.tensor(list(z), device=DEV) for z in (moves.keys(), moves.values()))
        a, b = (out.view(torch.uint8), x.view(torch.uint8)) if x.dtype == torch.float8_e4m3fn else (out, x)
        a[to] = b[frm]
    return out


def _same(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


EVICT_LENS = [[[0, 5, 300], [1, 1500, 64]], [[2000]], [[33] * 8] * 9]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("kv8", 64), ("kv8", 128), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 16])
def test_eviction_in_place(dtype, D, page):
    for seed, lens in enumerate(EVICT_LENS):
        for part in (0.0, 0.1, 0.5, 0.97, 1.0):
            s = Setup(lens, 2, D, dtype, page, seed=seed)
            keep, counts = _lists(s.lens_h, part, seed)
            after, moves, alone = C.evict(s.lens_h, keep, counts, s.row)
            w = torch.randn(s.n_rows, device=DEV)
            want = [_moved(x, moves) for x in (s.k, s.v, w)]
            bad = torch.zeros(1, dtype=torch.int32, device=DEV)
            lens_out = None if seed else torch.zeros_like(s.lens)
            F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), weights=w, lens_out=lens_out, bad=bad)
            assert all(_same(x, y) for x, y in zip((s.k, s.v, w), want)) and int(bad) == 0 and not alone
            assert (s.lens if lens_out is None else lens_out).flatten().tolist() == after.tolist()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("kv8", 64), ("kv8", 128), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("n_slots", [1, 4, 1000])
def test_eviction_in_place_however_the_rows_are_dealt(dtype, D, page, n_slots):
    """Whole rows, 64 bytes and 32 of them by a workgroup; lists of one run and of several, of a pair among wrong ones."""
    for lens, most in (([[9, 6000, 1], [0, 2500, 700]], 0.6), ([[300, 17, 1000]], 0.9), ([[5000]], 1.0)):
        s = Setup(lens, 2, D, dtype, page, seed=n_slots)
        keep, counts = _lists(s.lens_h, most, 3)
        if most == 0.6:
            keep[1, 1, 900] = keep[1, 1, 899]        # does not ascend, far behind the list's begin
        after, moves, alone = C.evict(s.lens_h, keep, counts, s.row)
        assert alone == ([4] if most == 0.6 else [])
        w = torch.randn(s.n_rows, device=DEV)
        want = [_moved(x, moves) for x in (s.k, s.v, w)]
        bad = torch.zeros(1, dtype=torch.int32, device=DEV)
        F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), weights=w, bad=bad, n_slots=n_slots)
        assert all(_same(x, y) for x, y in zip((s.k, s.v, w), want)) and int(bad) == len(alone)
        assert s.lens.flatten().tolist() == after.tolist()


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("kv8", 64), ("f32", 128)])
@pytest.mark.parametrize("page,to_page", [(0, 0), (16, 0), (0, 32), (64, 16)])
def test_eviction_into_another_cache(dtype, D, page, to_page):
    for seed, lens in enumerate(EVICT_LENS):
        s = Setup(lens, 2, D, dtype, page, seed=seed)
        keep, counts = _lists(s.lens_h, 0.4, seed)
        if seed == 1:                                # any order, and a row twice
            keep[0, 0, :counts[0, 0]] = np.random.default_rng(0).integers(0, 2000, counts[0, 0])
        to = Setup(counts, 3, D, dtype, to_page, seed=9)
        after, moves, alone = C.evict(s.lens_h, keep, counts, s.row, to.row, to.cap_h)
        w, w_to = torch.randn(s.n_rows, device=DEV), torch.zeros(to.n_rows, device=DEV)
        want = [_moved(x, moves, y) for x, y in ((s.k, to.k), (s.v, to.v), (w, w_to))]
        before, bad = s.k.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
        lens_out = s.lens if seed == 2 else torch.zeros_like(s.lens)
        F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), into=to.cache, lens_out=lens_out, weights=w, weights_out=w_to, bad=bad)
        assert all(_same(x, y) for x, y in zip((to.k, to.v, w_to), want)) and _same(s.k, before) and int(bad) == 0 and not alone
        assert lens_out.flatten().tolist() == after.tolist()


def test_lists_that_are_wrong_leave_their_pair_alone():
    for page in (0, 16):
        s = Setup([[20] * 8] * 2, 2, 64, page=page)
        keep, counts = _lists(s.lens_h, 0.5, 1)
        counts[:] = 6
        keep[:, :, :6] = [0, 3, 4, 9, 15, 19]
        keep[0, 0, 3] = 20                           # no token of the pair
        keep[0, 1, 0] = -1
        keep[0, 2, 2] = 3                            # twice
        keep[0, 3, 5] = 8                            # descends
        counts[0, 4] = -1
        counts[0, 5] = keep.shape[2] + 1
        keep[0, 6, 0] = -2 ** 31
        s.lens_h[1, 0] = -3
        s.lens_h[1, 1] = 5                           # shorter than its list says
        if page:
            s.pages[8 + 2, 0] = -1
        else:
            s.off[8 + 2] = s.n_rows - 10
        s.make()
        after, moves, alone = C.evict(s.lens_h, keep, counts, s.row)
        assert len(alone) == 10
        want = [_moved(x, moves) for x in (s.k, s.v)]
        bad = torch.zeros(1, dtype=torch.int32, device=DEV)
        F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), bad=bad)
        assert _same(s.k, want[0]) and _same(s.v, want[1]) and int(bad) == 10
        assert s.lens.flatten().tolist() == after.tolist()


def test_lists_that_are_wrong_into_another_cache():
    s, to = Setup([[20] * 6], 2, 64), Setup([[6] * 6], 0, 64, page=16)
    to.cap_h[0, 5] = 5                               # no room
    to.make()
    keep, counts = _lists(s.lens_h, 0.5, 1)
    counts[:] = 6
    keep[:, :, :6] = [4, 3, 3, 9, 15, 19]            # any order will do
    keep[0, 0, 3], keep[0, 1, 0], counts[0, 2] = 20, -1, -1
    after, moves, alone = C.evict(s.lens_h, keep, counts, s.row, to.row, to.cap_h)
    assert alone == [0, 1, 2, 5]
    out, bad = torch.full_like(s.lens, 77), torch.zeros(1, dtype=torch.int32, device=DEV)
    F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), into=to.cache, lens_out=out, bad=bad)
    assert out.flatten().tolist() == after.tolist() == [0, 0, 0, 6, 6, 0] and int(bad) == 4
    at = torch.tensor(list(moves.keys()), device=DEV)
    assert _same(to.k[at], s.k[torch.tensor(list(moves.values()), device=DEV)])


def test_into_other_pages_of_the_same_pool():
    s = Setup([[50, 20]], 0, 64, page=16, pool=8)
    free = sorted(set(range(s.n_rows // 16)) - set(s.pages.flatten().tolist()))[:4]
    to = F.Cache(s.k, s.v, I32([[32, 32]]), pages=I32(np.array(free).reshape(2, 2)), page_rows=16)
    keep, counts = _lists(s.lens_h, 0.4, 3)
    row_to = lambda p, t: S.row_of(p, t, s.n_rows, None, np.array(free).reshape(2, 2), 16)
    after, moves, _ = C.evict(s.lens_h, keep, counts, s.row, row_to, [[32, 32]])
    want = _moved(s.k, moves)
    out = torch.zeros_like(s.lens)
    F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), into=to, lens_out=out)
    assert _same(s.k, want) and out.flatten().tolist() == after.tolist()


# ---- together ----------------------------------------------------------------------------------------------
class Loop:
    """A step with a compression at its end: append, attend, add up the weights, select, evict in place."""

    def __init__(self, page=0, dtype="bf16", shared=True, D=64, G=4, q_len=3):
        self.s = s = Setup([[60, 90], [33, 40]], 40, D, dtype, page, scales=True)
        Hq = 2 * G
        g = torch.Generator().manual_seed(5)
        self.q, self.k_new, self.v_new = (torch.randn(2, q_len, h, D, generator=g).to(torch.bfloat16).to(DEV) for h in (Hq, 2, 2))
        self.out = torch.zeros(2, q_len, Hq, D, device=DEV)
        self.lse = torch.zeros(2, q_len, Hq, device=DEV)
        self.weights = torch.zeros(s.n_rows, device=DEV)
        self.ws = torch.zeros(F.fairkv_tree_workspace_bytes(s.cache, Hq, q_len), dtype=torch.uint8, device=DEV)
        self.ws2 = torch.zeros(F.fairkv_select_workspace_bytes(s.cache, shared), dtype=torch.uint8, device=DEV)
        self.budget = I32([100, 60]) if shared else I32([[50, 50], [30, 30]])
        self.keep, self.n_keep = torch.zeros(2, 2, 140, dtype=torch.int32, device=DEV), torch.zeros(2, 2, dtype=torch.int32, device=DEV)
        self.q_out, self.bad = torch.zeros_like(self.q), torch.zeros(1, dtype=torch.int32, device=DEV)
        self.scale = D ** -0.5

    def step(self, stream=None):
        s, kw = self.s, dict(stream=stream)
        F.fairkv_append_rotated(s.cache, s.lens, self.q, self.k_new, self.v_new, self.q_out, bad=self.bad, **kw)
        F.fairkv_decode_attn_tree(s.cache, s.lens, self.q_out, self.ws, self.out, self.lse, self.scale, **kw)
        F.fairkv_attn_weights(s.cache, s.lens, self.q_out, self.lse, self.weights, self.scale, decay=1.0, **kw)
        F.fairkv_select(s.cache, s.lens, self.weights, self.budget, self.keep, self.n_keep, self.ws2, pool=3, sink=2, recent=8, bad=self.bad, **kw)
        F.fairkv_evict(s.cache, s.lens, self.keep, self.n_keep, weights=self.weights, bad=self.bad, **kw)

    def state(self):
        s = self.s
        return [x.clone() for x in (s.k.view(torch.uint8), s.v.view(torch.uint8), s.lens, self.weights, self.out, self.keep, self.n_keep, self.bad)]


@pytest.mark.parametrize("page,dtype,shared", [(0, "bf16", True), (16, "bf16", False), (16, "kv8", True)])
def test_steps_of_a_compressed_cache(page, dtype, shared):
    a = Loop(page, dtype, shared)
    s = a.s
    for turn in range(4):
        lens = s.lens.cpu().numpy()
        a.step()
        assert int(a.bad) == 0
        after = s.lens.cpu().numpy()
        assert (after == a.n_keep.cpu().numpy()).all() and (after <= lens + 3).all()
        if shared:
            assert (after.sum(1) <= [100, 60]).all()
        else:
            assert (after <= [[50, 50], [30, 30]]).all()
        # of every query its weights sum up to 1 over the rows of its pair: before anything is dropped, after one step
        if turn == 0:
            kept = a.weights.double().cpu().numpy()
            for p in range(4):
                rows = [s.row(p, t) for t in range(int(after.reshape(-1)[p]))]
                assert 0 < kept[rows].sum() <= 3 * 4 * (1 + 1e-4)


def test_weights_of_the_attentions_own_lse_sum_to_the_queries():
    a = Loop(16)
    s = a.s
    F.fairkv_append_rotated(s.cache, s.lens, a.q, a.k_new, a.v_new, a.q_out)
    F.fairkv_decode_attn_tree(s.cache, s.lens, a.q_out, a.ws, a.out, a.lse, a.scale)
    F.fairkv_attn_weights(s.cache, s.lens, a.q_out, a.lse, a.weights, a.scale)
    for p in range(4):
        rows = [s.row(p, t) for t in range(int(s.lens.flatten()[p]))]
        # 12 queries, each off by what its scores are (64 products of a size below 8: 2^-15) and its lse (the same)
        assert abs(float(a.weights.double()[rows].sum()) - 12) <= 12 * 2.0 ** -14


def test_a_captured_step_of_a_compressed_cache():
    eager, captured = Loop(16), Loop(16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        captured.step()                              # warm
    side.synchronize()
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured.step()
    for turn in range(5):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        other = torch.randn(1000, device=DEV).sum()      # the program's own work in between
        assert all(torch.equal(x, y) for x, y in zip(eager.state(), captured.state())), turn
        assert math.isfinite(float(other))


def test_on_a_stream_of_the_callers():
    a, b = Loop(0), Loop(0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a.step()
    b.step(side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.state(), b.state()))


def test_two_captured_steps_that_share_a_workspace():
    """Two sequences of long rows, each with a graph of its own, replayed in turn on one stream over one workspace."""
    class Long:
        def __init__(self, seed):
            self.s = s = Setup([[9000, 7000]], 0, 64, page=64, seed=seed)
            self.w = torch.from_numpy(_some_weights(s.n_rows, seed, "tail")).to(DEV)
            self.keep, self.n_keep = torch.zeros(1, 2, 9000, dtype=torch.int32, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV)
            self.budget, self.bad = I32([14000]), torch.zeros(1, dtype=torch.int32, device=DEV)

        def step(self, ws):
            F.fairkv_select(self.s.cache, self.s.lens, self.w, self.budget, self.keep, self.n_keep, ws, pool=5, recent=16, bad=self.bad)
            F.fairkv_evict(self.s.cache, self.s.lens, self.keep, self.n_keep, weights=self.w, bad=self.bad)
            self.budget.sub_(1000)                   # a kernel of torch's, in the graph

    pairs = [(Long(1), Long(1)), (Long(2), Long(2))]     # eager, captured
    ws, eager_ws = (torch.zeros(F.fairkv_select_workspace_bytes(pairs[0][0].s.cache, True), dtype=torch.uint8, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    for eager, captured in pairs:
        with torch.cuda.stream(side):
            captured.step(ws)
        side.synchronize()
        eager.step(eager_ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            captured.step(ws)
        graphs.append(g)
    for turn in range(4):
        for g, (eager, captured) in zip(graphs, pairs):
            g.replay()
            eager.step(eager_ws)
        torch.cuda.synchronize()
        for eager, captured in pairs:
            for x, y in ((eager.s.k, captured.s.k), (eager.s.v, captured.s.v), (eager.w, captured.w), (eager.s.lens, captured.s.lens), (eager.n_keep, captured.n_keep)):
                assert torch.equal(x, y), turn
            assert int(captured.bad) == int(eager.bad) == 0
            assert int(captured.s.lens.sum()) == 14000 - 1000 * (turn + 1)


def test_rows_beyond_32_bits():
    """A pair at the end of a cache of 20 million rows: its bytes, and its weights' bytes, are beyond 32 bits."""
    n_rows, n, D = 20_000_000, 700, 128
    k = torch.empty(n_rows, D, dtype=torch.bfloat16, device=DEV)
    w, first = torch.zeros(n_rows, device=DEV), n_rows - n - 5
    g = torch.Generator().manual_seed(1)
    k[first:] = torch.randn(n_rows - first, D, generator=g).to(torch.bfloat16).to(DEV)
    q = torch.randn(1, 2, D, generator=g).to(torch.bfloat16).to(DEV)
    lens, off = I32([[n]]), torch.tensor([[first]], device=DEV)
    cache = F.Cache(k, k, I32([[n]]), off=off)
    near = F.Cache(k[first:].clone(), k[first:].clone(), I32([[n]]), off=torch.zeros_like(off))
    lse = torch.full((1, 2), 3.0, device=DEV)
    F.fairkv_attn_weights(cache, lens, q, lse, w, 0.1)
    w_near = torch.zeros(n_rows - first, device=DEV)
    F.fairkv_attn_weights(near, lens, q, lse, w_near, 0.1)
    assert torch.equal(w[first:], w_near) and float(w_near[:n].min()) > 0
    lists = []
    for c, x in ((cache, w), (near, w_near)):
        keep, n_keep = torch.zeros(1, 1, n, dtype=torch.int32, device=DEV), torch.zeros(1, 1, dtype=torch.int32, device=DEV)
        ws = torch.zeros(F.fairkv_select_workspace_bytes(c, False), dtype=torch.uint8, device=DEV)
        F.fairkv_select(c, lens, x, I32([[200]]), keep, n_keep, ws, recent=10)
        lists.append((keep, n_keep))
    assert all(torch.equal(x, y) for x, y in zip(*lists)) and int(lists[0][1]) == 200
    rows = (first + lists[0][0][0, 0, :200].long())
    want = k[rows].clone()
    out = torch.zeros_like(lens)
    small = F.Cache(torch.zeros(200, D, dtype=torch.bfloat16, device=DEV), torch.zeros(200, D, dtype=torch.bfloat16, device=DEV), I32([[200]]), off=torch.zeros_like(off))
    F.fairkv_evict(cache, lens, *lists[0], into=small, lens_out=out)
    assert torch.equal(small.k, want) and torch.equal(small.v, want)
    v = k[first:].clone()
    apart = F.Cache(k, k.clone(), I32([[n]]), off=off)
    F.fairkv_evict(apart, lens, *lists[0])
    assert torch.equal(k[first:first + 200], want) and torch.equal(k[first + 200:], v[200:]) and int(lens) == 200
