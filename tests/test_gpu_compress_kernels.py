"""Every kernel of the compression of a growing cache that a call can take, against the oracle: the widths of the attention weights in both types and sizes of
heads, selections and moves of more groups than slots, a group of more blocks than a workgroup looks at in one turn, and what lies behind a workspace."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import compress as C
from test_gpu_compress import _check_select, _lists, _lse, _moved, _same, _some_weights, _weight_tolerance, _words
from test_gpu_step import DEV, I32, Setup

pytestmark = pytest.mark.gpu


# ---- weights: up to 64, 128, 256 columns in LDS, and 512 (heads of 128) or 1024 (of 64) ----
@pytest.mark.parametrize("dtype", ["bf16", "kv8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,n", [(5, 13), (16, 8), (3, 43), (8, 32), (9, 29), (16, 32), (13, 50), (16, 64)])
@pytest.mark.parametrize("tree,ragged", [(False, False), (True, True)])
def test_weights_of_every_width(dtype, D, G, n, tree, ragged):
    """65, 128, 129, 256, 261, 512, 650 and 1024 columns; runs that end in a turn of few tiles, which several waves share."""
    s = Setup([[n + 300, 33 + n], [n, 290]], 3, D, dtype, page=16 if tree else 0, seed=n, scales=True)
    rng = np.random.default_rng(n + D)
    B, Hq, scale = 2, 2 * G, 1.0 / math.sqrt(D)
    n_new = np.array([n - 2, n // 2]) if ragged else np.full(B, n)
    words = _words(B, n, n) if tree else None
    q = torch.randn(B, n, Hq, D, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16)
    q_h = q.double().numpy()
    lse = _lse(s, q_h, scale, n_new, words).astype(np.float32)
    old = np.exp(rng.standard_normal(s.n_rows)).astype(np.float32)
    want = C.attn_weights(q_h, s.numbers()[0], s.lens_h, lse, old, scale, 0.75, n_new, words, s.row, s.ks)
    tol = _weight_tolerance(s, q_h, lse.astype(np.float64), scale, n_new, words, old, 0.75, want)
    kw = dict(tree=None if words is None else torch.from_numpy(words.view(np.int64)).to(DEV), n_new=I32(n_new) if ragged else None, decay=0.75)
    first = None
    for n_slots in (None, 1):                        # a tile a workgroup, shared by its waves; all of them in one
        out = torch.from_numpy(old).to(DEV)
        F.fairkv_attn_weights(s.cache, s.lens, q.to(DEV), torch.from_numpy(lse).to(DEV), out, scale, n_slots=n_slots, **kw)
        off = np.abs(out.double().cpu().numpy() - want)
        assert (off <= tol).all(), (np.max(off / tol), np.argmax(off / tol))
        first = out if first is None else first
        assert torch.equal(out, first)


# ---- select ----
@pytest.mark.parametrize("kind", ["tail", "few", "signs"])
@pytest.mark.parametrize("pool", [1, 7])
@pytest.mark.parametrize("page", [0, 16])
def test_more_groups_than_slots(page, pool, kind):
    """As many workgroups as a batch has: the narrower ones, which alone have groups of up to 7680 rows in a launch without large ones."""
    rng = np.random.default_rng(3)
    s = Setup(rng.integers(0, 130, (9, 6)), 0, 64, page=page, seed=2)
    w = _some_weights(s.n_rows, 3, kind)
    for n_slots in (1, 8, 53):
        for shared in (True, False):
            total = s.lens_h.sum(1) if shared else s.lens_h
            for part, sink, recent in ((0.5, 0, 0), (0.3, 4, 8), (0.0, 0, 5), (2.0, 1, 0)):
                _check_select(s, w, np.rint(total * part), shared, pool, sink, recent, n_slots=n_slots)


@pytest.mark.parametrize("shared", [True, False])
def test_a_packed_batch_of_short_pairs(shared):
    """A pair could have all of a packed cache's rows, so the launch has room for large groups, of which there are none."""
    s = Setup(np.random.default_rng(5).integers(0, 260, (24, 8)), 0, 64, seed=2)
    assert s.n_rows > 20000
    total = s.lens_h.sum(1) if shared else s.lens_h
    for kind, part, pool in (("tail", 0.5, 1), ("few", 0.25, 7), ("signs", 0.9, 63)):
        _check_select(s, _some_weights(s.n_rows, 3, kind), np.rint(total * part), shared, pool, 2, 8)


@pytest.mark.parametrize("pool", [1, 5])
def test_groups_of_many_rows_and_more_of_them_than_slots(pool):
    s = Setup([[3500, 100], [7000, 1], [40, 3000]], 0, 64, page=16, seed=4, pool=0)
    cache = F.Cache(s.k, s.v, I32(s.cap_h), pages=I32(s.pages), page_rows=16)
    assert cache.struct.max_pages * 16 <= 7680       # a pair's own budget: no group can be a large one
    w = _some_weights(s.n_rows, 3, "near")
    for n_slots in (1, 5, 6):
        _check_select(s, w, np.rint(s.lens_h * 0.4), False, pool, 2, 16, n_slots=n_slots)


def _chosen(w, lens, off, budget, pool, sink, recent):
    """The selection of one group by a stable sort; a pair's rows follow one another."""
    keys, pairs, tokens, stay = [], [], [], []
    for p, n in enumerate(lens):
        x = w[off[p]:off[p] + n]
        first, end = min(sink, n), max(min(sink, n), n - min(recent, n))
        c = x[first:end]
        best = c.copy()
        for d in range(1, pool // 2 + 1):
            best[d:] = np.maximum(best[d:], c[:-d])
            best[:-d] = np.maximum(best[:-d], c[d:])
        keys.append(best), pairs.append(np.full(best.size, p)), tokens.append(np.arange(first, end))
        stay.append(np.r_[0:first, end:n])
    room = max(0, budget - sum(x.size for x in stay))
    keys, pairs, tokens = (np.concatenate(x) for x in (keys, pairs, tokens))
    at = np.argsort(-keys, kind="stable")[:room]     # in the order of heads and tokens where values are equal
    return [np.sort(np.concatenate([stay[p], tokens[at[pairs[at] == p]]])) for p in range(len(lens))]


@pytest.mark.parametrize("kind,pool", [("few", 1), ("tail", 5), ("near", 3)])
def test_a_group_of_more_blocks_than_a_workgroup_looks_at_in_one_turn(kind, pool):
    """The counts in front of a block are read 512 at a time: 548 blocks of 4096 rows, and ties all along."""
    lens, D = [560_000, 9, 561_111, 559_999, 560_001], 64
    off = np.concatenate([[0], np.cumsum(np.array(lens) + 3)[:-1]])
    n_rows = int(off[-1]) + lens[-1]
    w = _some_weights(n_rows, 7, kind)
    k = torch.zeros(n_rows, D, dtype=torch.bfloat16, device=DEV)
    cache = F.Cache(k, k, I32([lens]), off=torch.tensor(off[None], device=DEV))
    ws = torch.zeros(F.fairkv_select_workspace_bytes(cache, True), dtype=torch.uint8, device=DEV)
    for part in (0.02, 0.6, 0.97):
        budget = int(sum(lens) * part)
        keep, n_keep = torch.full((1, 5, max(lens)), -9, dtype=torch.int32, device=DEV), torch.zeros(1, 5, dtype=torch.int32, device=DEV)
        F.fairkv_select(cache, I32([lens]), torch.from_numpy(w).to(DEV), I32([budget]), keep, n_keep, ws, pool=pool, sink=4, recent=33)
        want = _chosen(w, lens, off, budget, pool, 4, 33)
        assert n_keep.flatten().tolist() == [x.size for x in want] and int(n_keep.sum()) == budget
        got = keep.cpu().numpy()[0]
        for p, x in enumerate(want):
            assert np.array_equal(got[p, :x.size], x) and (got[p, x.size:] == -9).all(), p


@pytest.mark.parametrize("shared", [True, False])
def test_what_lies_behind_a_workspace(shared):
    """A workspace of just the bytes it takes, in a larger buffer: large groups, small ones beside them, pairs that share rows, lengths that are none."""
    s = Setup([[30000, 9000], [40, 12000]], 0, 64, page=64, seed=1)
    need = F.fairkv_select_workspace_bytes(s.cache, shared)
    room = torch.full((need + (1 << 20),), 7, dtype=torch.uint8, device=DEV)
    ws = room[:need]
    ws.zero_()
    w = torch.from_numpy(_some_weights(s.n_rows, 2, "tail")).to(DEV)
    budget = I32([9000, 4000]) if shared else I32([[7000, 2000], [20, 4000]])
    same_rows = F.Cache(s.k, s.v, I32(s.cap_h), pages=I32(np.repeat(s.pages[:1], 4, 0)), page_rows=64)
    for cache, lens in ((s.cache, s.lens_h), (same_rows, [[30000] * 2] * 2), (s.cache, [[2 ** 31 - 1, -1], [2 ** 31 - 1, 7]]), (s.cache, s.lens_h)):
        keep, n_keep = torch.zeros(2, 2, 20000, dtype=torch.int32, device=DEV), torch.full((2, 2), -7, dtype=torch.int32, device=DEV)
        F.fairkv_select(cache, I32(lens), w, budget, keep, n_keep, ws, pool=3)
        assert bool((room[need:] == 7).all()) and not int(ws[:need // 3].max()) and bool((n_keep > -7).all())
    assert n_keep.sum(1).tolist() == ([9000, 4000] if shared else [9000, 4020])


# ---- evict: blocks of 64 entries, where there are many ----
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("kv8", 64), ("kv8", 128), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page,to_page", [(0, 0), (16, 32), (64, 0)])
def test_eviction_into_another_cache_of_many_blocks(dtype, D, page, to_page):
    for n_slots, lens, part in ((1, [[0, 5, 900], [1, 1500, 64]], 0.6), (1, [[130] * 8] * 5, 0.5), (2, [[5000]], 0.97)):
        s = Setup(lens, 2, D, dtype, page, seed=n_slots)
        keep, counts = _lists(s.lens_h, part, 3)
        assert keep[..., 0].size * -(-keep.shape[2] // 64) > 32 * n_slots
        if n_slots == 2:                             # any order, and a row twice
            keep[0, 0, :counts[0, 0]] = np.random.default_rng(0).integers(0, 5000, counts[0, 0])
        to = Setup(counts, 3, D, dtype, to_page, seed=9)
        after, moves, alone = C.evict(s.lens_h, keep, counts, s.row, to.row, to.cap_h)
        w, w_to = torch.randn(s.n_rows, device=DEV), torch.zeros(to.n_rows, device=DEV)
        want = [_moved(x, moves, y) for x, y in ((s.k, to.k), (s.v, to.v), (w, w_to))]
        bad, lens_out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros_like(s.lens)
        F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), into=to.cache, lens_out=lens_out, weights=w, weights_out=w_to, bad=bad, n_slots=n_slots)
        assert all(_same(x, y) for x, y in zip((to.k, to.v, w_to), want)) and int(bad) == 0 and not alone
        assert lens_out.flatten().tolist() == after.tolist()


def test_wrong_lists_into_another_cache_of_many_blocks():
    s, to = Setup([[400] * 8], 2, 64, page=16), Setup([[300] * 8], 0, 64)
    to.cap_h[0, 5] = 299                             # no room
    to.make()
    keep, counts = _lists(s.lens_h, 0.5, 1)
    counts[:] = 300
    keep = np.tile(np.arange(399, 99, -1, dtype=np.int32), (1, 8, 1))
    keep[0, 0, 280], keep[0, 1, 0], counts[0, 2] = 400, -1, 301
    after, moves, alone = C.evict(s.lens_h, keep, counts, s.row, to.row, to.cap_h)
    assert alone == [0, 1, 2, 5]
    k_before = to.k.clone()
    out, bad = torch.full_like(s.lens, 77), torch.zeros(1, dtype=torch.int32, device=DEV)
    F.fairkv_evict(s.cache, s.lens, I32(keep), I32(counts), into=to.cache, lens_out=out, bad=bad, n_slots=1)
    assert out.flatten().tolist() == after.tolist() and int(bad) == 4
    at = torch.tensor(list(moves.keys()), device=DEV)
    assert _same(to.k[at], s.k[torch.tensor(list(moves.values()), device=DEV)])
    mine = {to.row(p, i) for p in range(8) for i in range(300)}
    rest = [r for r in range(to.n_rows) if r not in mine]
    assert _same(to.k[rest], k_before[rest])
