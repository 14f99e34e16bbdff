"""Selection on the GPU over tokens that have no row in the cache: groups whose lengths add up to more than the cache's rows.  Such tokens do not stay and take no
part; everything else is the oracle's, exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import compress as C
from test_gpu_compress import _check_select, _some_weights
from test_gpu_step import DEV, I32, Setup

pytestmark = pytest.mark.gpu


def _holes(lens, page, share, seed, **kw):
    """A paged cache of whose pages a share is in the pool, and no more of them than the pool's; the others are none."""
    lens = np.asarray(lens)
    s = Setup(np.minimum(lens, page), 0, 64, page=page, seed=seed, **kw)      # a page each, to begin with
    rng = np.random.default_rng(seed)
    need = -(-lens // page).reshape(-1)
    total = max(1, int(need.sum() * share))
    s.n_rows = total * page
    s.k = torch.zeros(s.n_rows, 64, dtype=torch.bfloat16, device=DEV)
    s.v = s.k.clone()
    s.pages = np.full((need.size, int(need.max())), -1, dtype=np.int32)
    slots = [(p, i) for p in range(need.size) for i in range(need[p])]
    for page_id, at in zip(rng.permutation(total), rng.permutation(len(slots))[:total]):
        s.pages[slots[at]] = page_id
    s.lens_h, s.cap_h = lens.astype(np.int64), lens
    return s.make()


@pytest.mark.parametrize("kind", ["tail", "few", "signs"])
@pytest.mark.parametrize("lens,page,share,n_slots", [
    ([[2000] * 8], 16, 0.2, None),                   # a workgroup's by the rows, four times as long by its tokens
    ([[2000] * 8] * 5, 16, 0.2, 2),                  # more groups than slots: narrower workgroups
    ([[9000, 3000, 1, 0], [40, 12000, 7000, 90]], 32, 0.3, None),
    ([[30000, 1000], [20000, 17000], [5, 6]], 64, 0.1, 3),
    ([[70000, 60000], [30000, 80000]], 64, 0.35, None)])      # as many blocks as no workspace has
def test_groups_longer_than_the_cache_has_rows(lens, page, share, n_slots, kind):
    s = _holes(lens, page, share, 1)
    w = _some_weights(s.n_rows, 3, kind)
    there = np.array([sum(s.row(p, t) is not None for t in range(int(n))) for p, n in enumerate(s.lens_h.reshape(-1))]).reshape(s.lens_h.shape)
    for shared in (True, False):
        rows = there.sum(1) if shared else there
        for part, pool, sink, recent in ((0.4, 1, 0, 0), (0.1, 5, 4, 200), (1.5, 3, 0, 0), (0.0, 1, 3, 9)):
            _check_select(s, w, np.rint(rows * part), shared, pool, sink, recent, n_slots=n_slots)


def test_windows_over_tokens_without_rows():
    s = _holes([[3000] * 4], 16, 0.4, 2)
    w = _some_weights(s.n_rows, 3, "tail")
    _check_select(s, w, [900], True, 63, 2, 100)
    _check_select(s, w, [[200] * 4], False, 31, 0, 31)
    _check_select(s, w, [900], True, 3, 0, 0, max_keep=100)


def test_old_pages_that_were_given_back():
    """A window of every sequence is left, as long sequences have it whose first pages others were given."""
    B, H, n, page, left = 3, 2, 20000, 32, 40
    s = _holes([[n] * H] * B, page, left / (n // page), 1)
    s.pages[:] = -1
    s.pages[:, n // page - left:] = np.random.default_rng(0).permutation(B * H * left).reshape(B * H, left)
    s.make()
    w = _some_weights(s.n_rows, 3, "tail")
    for shared in (True, False):
        _check_select(s, w, np.full(B if shared else (B, H), 700), shared, 7, 16, 64)


@pytest.mark.parametrize("shared", [True, False])
def test_a_length_that_is_none_beside_healthy_groups(shared):
    """A packed cache, and one length as long as a number can be: the other groups are what they are without it."""
    B, H = 4, 2
    s = Setup(np.random.default_rng(0).integers(9000, 16000, (B, H)), 0, 64, seed=3)
    w = _some_weights(s.n_rows, 3, "tail")
    budget = np.rint((s.lens_h.sum(1) if shared else s.lens_h) * 0.3)
    most = 16000
    lists, counts = C.select(w.astype(np.float64), s.lens_h, budget, shared, 5, 4, 32, most, s.row)
    for p in (0, 3, B * H - 1):
        lens = s.lens_h.copy()
        lens.reshape(-1)[p] = 2 ** 31 - 1
        keep, n_keep = torch.full((B, H, most), -9, dtype=torch.int32, device=DEV), torch.full((B, H), -7, dtype=torch.int32, device=DEV)
        ws = torch.zeros(F.fairkv_select_workspace_bytes(s.cache, shared), dtype=torch.uint8, device=DEV)
        F.fairkv_select(s.cache, I32(lens), torch.from_numpy(w).to(DEV), I32(budget), keep, n_keep, ws, pool=5, sink=4, recent=32)
        others = [x for x in range(B * H) if (x // H != p // H if shared else x != p)]
        got, n = keep.cpu().numpy().reshape(-1, most), n_keep.flatten().tolist()
        for x in others:
            assert n[x] == len(lists[x]) and got[x, :n[x]].tolist() == lists[x], (p, x)
        assert not int(ws[:ws.numel() // 3].max())


def test_pairs_that_share_rows_within_what_the_cache_has():
    """Each has its own choice of them."""
    s = _holes([[1500] * 6], 16, 1.0, 5)
    s.pages[3:] = s.pages[:3]
    s.make()
    w = _some_weights(s.n_rows, 3, "tail")
    _check_select(s, w, [3000], True, 3, 1, 4)


def test_a_captured_selection_of_a_group_without_a_place():
    s = _holes([[70000, 60000], [30000, 80000]], 64, 0.35, 1)
    budget, w = I32([9000, 9000]), torch.from_numpy(_some_weights(s.n_rows, 3, "tail")).to(DEV)
    make = lambda: (torch.zeros(2, 2, 9000, dtype=torch.int32, device=DEV), torch.zeros(2, 2, dtype=torch.int32, device=DEV))
    ws = torch.zeros(F.fairkv_select_workspace_bytes(s.cache, True), dtype=torch.uint8, device=DEV)
    want, got = make(), make()
    run = lambda out: F.fairkv_select(s.cache, s.lens, w, budget, *out, ws, pool=3, recent=5)
    run(want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run(got)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(got)
    for turn in range(4):
        budget.sub_(500), w.mul_(0.5)
        run(want)
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        n = want[1]
        assert torch.equal(n, got[1]) and int(n.sum()) == 2 * (9000 - 500 * (turn + 1))
        assert all(torch.equal(want[0][b, h, :n[b, h]], got[0][b, h, :n[b, h]]) for b in range(2) for h in range(2))
