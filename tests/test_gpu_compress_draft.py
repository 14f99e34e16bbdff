"""Drafts and the compression of a growing cache on the GPU: weights follow the rows that an accept moves, a draft is scored behind its accept or in front of it,
and rows that were appended without being scored.  Moves and selections are exact; weights within the bounds of test_gpu_compress.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import compress as C
from oracle import step as S
from test_gpu_compress import _moved, _same, _weight_tolerance, _words
from test_gpu_step import DEV, I32, Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("kv8", 64), ("kv8", 128), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("q_len,page", [(1, 0), (3, 16), (17, 32), (64, 0)])
def test_weights_move_with_the_rows_of_an_accepted_path(dtype, D, q_len, page):
    rng = np.random.default_rng(q_len + D)
    B, Hkv = 7, 3
    n_new = rng.integers(0, q_len + 1, B)
    n_new[0] = q_len
    s = Setup(rng.integers(0, 80, (B, Hkv)) + n_new[:, None], 0, D, dtype, page, seed=q_len)
    path, n_path = np.full((B, q_len), -9), rng.integers(0, n_new + 1)
    n_path[0] = q_len
    for b in range(B):                       # any order, the same row twice
        path[b, :n_path[b]] = rng.integers(0, max(n_new[b], 1), n_path[b]) if b % 2 else np.sort(rng.permutation(n_new[b])[:n_path[b]])
    path[0] = np.arange(q_len)[::-1]
    if q_len > 1:
        n_path[1] = n_new[1] + 1             # left alone
    w = torch.randn(s.n_rows, device=DEV)
    want, moves, alone = S.accept(s.lens_h, path, n_path, n_new, Hkv, s.row)
    after = [_moved(x, moves) for x in (s.k, s.v, w)]
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    F.fairkv_accept(s.cache, s.lens, I32(path), I32(n_path), n_new=I32(n_new), bad=bad, weights=w)
    assert s.lens.cpu().numpy().reshape(-1).tolist() == want.tolist() and int(bad) == len(alone)
    assert all(_same(x, y) for x, y in zip((s.k, s.v, w), after))


class Draft:
    """Trees of 9 nodes over two sequences, of which one path is accepted."""
    PATHS, N_NEW = [[0, 2, 5, 7], [1, 3, 4, 8]], [9, 9]

    def __init__(self, dtype, page, D=64, G=4):
        self.s = s = Setup([[160, 90], [133, 340]], 60, D, dtype, page, scales=True)
        self.n, self.G, Hq = 9, G, 2 * G
        g = torch.Generator().manual_seed(3)
        self.q, self.k_new, self.v_new = (torch.randn(2, self.n, h, D, generator=g).to(torch.bfloat16).to(DEV) for h in (Hq, 2, 2))
        parents = [[-1, -1, 0, 1, 3, 2, 2, 5, 4], [-1, -1, 0, 1, 3, 2, 0, 5, 4]]
        self.words = np.zeros((2, self.n), dtype=np.uint64)
        for b in range(2):
            for i, up in enumerate(parents[b]):
                self.words[b, i] = (self.words[b, up] if up >= 0 else np.uint64(0)) | np.uint64(1 << i)
        self.tree = torch.from_numpy(self.words.view(np.int64)).to(DEV)
        self.path, self.n_path = I32([p + [-1] * 5 for p in self.PATHS]), I32([4, 4])
        self.out, self.lse, self.q_out = torch.zeros(2, self.n, Hq, D, device=DEV), torch.zeros(2, self.n, Hq, device=DEV), torch.zeros_like(self.q)
        self.ws = torch.zeros(F.fairkv_tree_workspace_bytes(s.cache, Hq, self.n), dtype=torch.uint8, device=DEV)
        self.scale = D ** -0.5
        self.weights = torch.rand(s.n_rows, generator=g).to(DEV)
        F.fairkv_append_rotated(s.cache, s.lens, self.q, self.k_new, self.v_new, self.q_out)
        F.fairkv_decode_attn_tree(s.cache, s.lens, self.q_out, self.ws, self.out, self.lse, self.scale, tree=self.tree)
        s.lens_h = s.lens.cpu().numpy().astype(np.int64)

    def wanted(self, q, lse, n_new, words, old, decay):
        """The oracle's weights, and how far they may be off, of the cache as it is."""
        s = self.s
        q, lse, old = q.double().cpu().numpy(), lse.double().cpu().numpy(), old.double().cpu().numpy()
        want = C.attn_weights(q, s.numbers()[0], s.lens_h, lse, old, self.scale, decay, n_new, words, s.row, s.ks)
        return want, _weight_tolerance(s, q, lse, self.scale, n_new, words, old, decay, want)

    def compress(self):
        """Select and evict in place, against the oracle on the weights as they are."""
        s = self.s
        w = self.weights.cpu().numpy()
        lists, counts = C.select(w.astype(np.float64), s.lens_h, [150, 200], True, 3, 2, 8, 400, s.row)
        keep, n_keep = torch.full((2, 2, 400), -5, dtype=torch.int32, device=DEV), torch.zeros(2, 2, dtype=torch.int32, device=DEV)
        ws = torch.zeros(F.fairkv_select_workspace_bytes(s.cache, True), dtype=torch.uint8, device=DEV)
        F.fairkv_select(s.cache, s.lens, self.weights, I32([150, 200]), keep, n_keep, ws, pool=3, sink=2, recent=8)
        assert n_keep.cpu().numpy().tolist() == counts.tolist()
        got = keep.cpu().numpy().reshape(4, -1)
        assert all(got[p, :len(x)].tolist() == x for p, x in enumerate(lists))
        _, moves, _ = C.evict(s.lens_h, got.reshape(2, 2, -1), counts, s.row)
        want = [_moved(x, moves) for x in (s.k, s.v, self.weights)]
        F.fairkv_evict(s.cache, s.lens, keep, n_keep, weights=self.weights)
        assert all(_same(x, y) for x, y in zip((s.k, s.v, self.weights), want)) and s.lens.cpu().numpy().tolist() == counts.tolist()


FORMS = [("bf16", 0), ("bf16", 16), ("kv8", 16)]


@pytest.mark.parametrize("dtype,page", FORMS)
def test_a_draft_that_is_scored_behind_its_accept(dtype, page):
    d = Draft(dtype, page)
    s = d.s
    F.fairkv_accept(s.cache, s.lens, d.path, d.n_path)
    s.lens_h = s.lens.cpu().numpy().astype(np.int64)
    assert s.lens_h.tolist() == [[164, 94], [137, 344]]
    at = torch.tensor(d.PATHS, device=DEV)
    q, lse = (torch.stack([x[b, at[b]] for b in range(2)]) for x in (d.q_out, d.lse))
    old = d.weights.clone()
    want, tol = d.wanted(q, lse, [4, 4], None, old, 0.9)
    F.fairkv_attn_weights(s.cache, s.lens, q, lse, d.weights, d.scale, decay=0.9)
    assert (np.abs(d.weights.double().cpu().numpy() - want) <= tol).all()
    # what the accepted queries gave sums up to one for each of them: all that they see is still there
    for p in range(4):
        rows = [s.row(p, t) for t in range(int(s.lens_h.reshape(-1)[p]))]
        gave = want[rows].sum() - 0.9 * old.double().cpu().numpy()[rows[:-4]].sum()
        assert abs(gave - 4 * d.G) <= 4 * d.G * 2.0 ** -14      # 64 products of scores below 8, and the lse's own (the same)
    d.compress()


@pytest.mark.parametrize("dtype,page", FORMS)
def test_a_draft_that_is_scored_in_front_of_its_accept(dtype, page):
    d = Draft(dtype, page)
    s = d.s
    want, tol = d.wanted(d.q_out, d.lse, d.N_NEW, d.words, d.weights, 0.9)
    F.fairkv_attn_weights(s.cache, s.lens, d.q_out, d.lse, d.weights, d.scale, tree=d.tree, decay=0.9)
    _, moves, alone = S.accept(s.lens_h, [p + [-1] * 5 for p in d.PATHS], [4, 4], d.N_NEW, 2, s.row)
    assert not alone and moves
    for x in (want, tol):
        before = x.copy()
        for to, source in moves.items():
            x[to] = before[source]
    F.fairkv_accept(s.cache, s.lens, d.path, d.n_path, weights=d.weights)
    s.lens_h = s.lens.cpu().numpy().astype(np.int64)
    assert (np.abs(d.weights.double().cpu().numpy() - want) <= tol).all()
    d.compress()


def test_rows_that_were_appended_and_not_scored_have_what_was_there():
    """Behind the rows that stay lie weights of dropped ones: a step that is not scored leaves them to its tokens, one that is starts its own from 0."""
    for page in (0, 16):
        s = Setup([[50, 40]], 30, 64, page=page)
        w = torch.rand(s.n_rows, generator=torch.Generator().manual_seed(1)).to(DEV) + 1
        keep = I32(np.arange(10, 30)[None, None].repeat(2, 1))
        before = w.clone()
        F.fairkv_evict(s.cache, s.lens, keep, I32([[20, 20]]), weights=w)
        rows = lambda p, *t: [s.row(p, x) for x in range(*t)]
        for p in range(2):
            assert torch.equal(w[rows(p, 20)], before[rows(p, 10, 30)]) and torch.equal(w[rows(p, 20, 40)], before[rows(p, 20, 40)])
        g = torch.Generator().manual_seed(2)
        new = lambda n, h: torch.randn(1, n, h, 64, generator=g).to(torch.bfloat16).to(DEV)
        for scored in (False, True):
            q = new(3, 4)
            F.fairkv_append_rotated(s.cache, s.lens, q, new(3, 2), new(3, 2), q)
            if scored:
                stale, first = w.clone(), w.clone()
                for p in range(2):
                    first[rows(p, 20, 23)] = 0      # what a caller does with the step that is not scored
                lse = torch.full((1, 3, 4), 5.0, device=DEV)
                zero = torch.zeros_like(w)
                for x in (stale, first, zero):
                    F.fairkv_attn_weights(s.cache, s.lens, q, lse, x, 0.125, decay=1.0)
                for p in range(2):
                    unscored, own = rows(p, 20, 23), rows(p, 23, 26)
                    assert torch.equal(stale[own], zero[own]) and torch.equal(first[unscored], zero[unscored])
                    assert torch.equal(stale[unscored], w[unscored] + zero[unscored]) and bool((stale[unscored] > 1).all())
