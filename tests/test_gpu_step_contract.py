"""What the header promises of a step over a growing cache, at every width that the attention's columns can be dealt in and for inputs of any
value.  Against the oracle, with the tolerances that test_gpu_step.py derives where no others stand beside a test."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from oracle import step as S
from test_gpu_step import DEV, I32, Setup, _attend, _compare, _random_tree

pytestmark = pytest.mark.gpu

# Drafts of 8 heads a KV head in 1, 2, 4 and 8 waves side by side, for the pairs below and one workgroup (two blocks of it at the last)
WIDTHS = [4, 8, 16, 40]


@pytest.mark.parametrize("n_slots", [1, 16])
@pytest.mark.parametrize("q_len", WIDTHS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "kv8"])
@pytest.mark.parametrize("page", [0, 16])
def test_rows_that_the_cache_does_not_have_at_every_width(page, dtype, D, q_len, n_slots):
    s = Setup([[300, 140], [190, 164]], 1, D, dtype, page, seed=6, scales=True)
    if page:
        s.pages[0, 2], s.pages[1, 0], s.pages[2, 5], s.pages[3, 1] = -1, 1 << 30, s.n_rows // page, -(1 << 31)
    else:
        s.off[0], s.off[3] = s.n_rows - 299, -1
        row = s.row
        s.row = lambda p, t: None if p in (0, 3) else row(p, t)      # a run that does not fit is not read at all
    s.make()
    for out_dtype in (torch.float32, torch.bfloat16):
        _compare(s, *_attend(s, 16, q_len, out_dtype, n_slots=n_slots), None, None)


@pytest.mark.parametrize("n_slots", [None, 1, 16])
@pytest.mark.parametrize("G,q_len", [(1, 1)] + [(8, n) for n in WIDTHS])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 0)])
def test_infinite_values_in_front_of_the_draft(D, page, G, q_len, n_slots):
    """Every node sees them: the output is that infinity, whatever the weight's bits, the width and the type of the output."""
    s = Setup(np.array([[333, 70], [45, 700]]) + q_len, 1, D, "bf16", page, seed=3)
    for p in range(4):
        for i, t in enumerate((0, 5, 31, 40)):                       # before a draft of pair 2, which has 45 rows in front of it
            s.v[s.row(p, t), 3 * i + p] = math.inf if i % 2 else -math.inf
    tree = _random_tree(2, q_len, np.random.default_rng(4))
    for out_dtype in (torch.float32, torch.bfloat16):
        _compare(s, *_attend(s, 2 * G, q_len, out_dtype, tree, n_slots=n_slots), tree, None)


@pytest.mark.parametrize("n_slots", [1, 8])
@pytest.mark.parametrize("q_len", [1] + WIDTHS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_an_infinite_value_under_small_weights(out_dtype, q_len, n_slots):
    """Row 0 of each pair has the largest score, all others lie `gap` log2 units below it; rows 1 and 40 have an infinite V.  Weights of 2**-gap
    that are bf16 numbers themselves, and some that are not."""
    gaps = [1, 7, 60, 100.5, 110, 111, 111.5, 112, 112.5, 113, 118, 120.5, 125]
    B = len(gaps)
    s = Setup(np.full((B, 1), 96 + q_len), 0, 128, seed=5)
    s.k.zero_(), s.v.fill_(1.0)
    for p, gap in enumerate(gaps):
        rows = [s.row(p, t) for t in range(96 + q_len)]
        s.k[rows[1:], 0] = -gap
        s.v[rows[1], 5], s.v[rows[40], 9] = math.inf, -math.inf
    q = torch.zeros((B, q_len, 8, 128), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1
    out = _attend(s, 8, q_len, out_dtype, n_slots=n_slots, q=q, scale=math.log(2.0))[1].double().cpu().numpy()
    assert np.isposinf(out[..., 5]).all() and np.isneginf(out[..., 9]).all()
    # out is a mean of ones: 2^-16 of each weight at most are lost, 136 fp32 sums 2^-24 each; a bf16 number next to 1 is 2^-8 away
    assert np.abs(np.delete(out, [5, 9], axis=-1) - 1).max() <= (2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -16 + 136 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["bf16", "kv8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("expected", [1, 20000, 60000, 1 << 40])
def test_rows_that_are_expected_cost_no_bits_of_a_bf16_output(expected, D, dtype):
    """256 columns in one, two, four and eight waves side by side: a weight is off by 2^-16 of itself in all of them."""
    s = Setup(np.random.default_rng(9).integers(20, 60, (4, 2)) + 32, 20000, D, dtype, seed=9, scales=True)
    kw = dict(k_scale=s.ks.tolist(), v_scale=s.vs.tolist()) if dtype == "kv8" else {}
    s.cache = F.Cache(s.k, s.v, I32(s.cap_h), expected_rows=expected, off=torch.as_tensor(s.off.reshape(4, 2), device=DEV), **kw)
    q, out, lse, scale = _attend(s, 16, 32, torch.bfloat16, n_slots=64)
    _compare(s, q, out, lse, scale, None, None)
    q_h = q.float().cpu().numpy().astype(np.float64).reshape(4, 32, 2, 8, D) * s.ks[None, None, :, None, None]
    vs = np.repeat(s.vs, 8)[None, None, :]
    ref, _, v_top, s_top = S.attend(q_h.reshape(4, 32, 16, D), *s.numbers(), s.lens_h, [32] * 4, lambda b, i, j: j <= i, scale, 2, s.row)
    ref, v_top = ref * vs[..., None], v_top * vs
    # scores: D products in fp32, twice for the sum; the weights' bits; 92 fp32 sums; the output's own rounding
    tol = (2 * (s_top * D * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -16 + 92 * 2.0 ** -24) * v_top
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol[..., None] + 2.0 ** -8 * (np.abs(ref) + tol[..., None])).all()


@pytest.mark.parametrize("scales", [7.0, 0.02, 0.3, [1.0, 0.033], [448.0, 3e-3]])
def test_8_bit_rows_are_the_quotient_rounded_to_nearest_even(scales):
    """Every bf16 number as a value: the bytes of x / scale in fp32, rounded to E4M3, beyond +-448 as +-448."""
    H = np.size(scales)
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).view(8, 64, 1, 128)
    v_new = every.expand(8, 64, H, 128).contiguous()
    n_rows = 8 * H * 64
    k, v = (torch.zeros(n_rows, 128, dtype=torch.uint8, device=DEV) for _ in range(2))
    off = torch.arange(8 * H, device=DEV).view(8, H) * 64
    cache = F.Cache(k, v, I32(np.full((8, H), 64)), off=off, k_scale=scales, v_scale=scales)
    q = torch.zeros(8, 64, H, 128, dtype=torch.bfloat16, device=DEV)
    F.fairkv_append_rotated(cache, I32(np.zeros((8, H))), q, v_new.to(DEV), v_new.to(DEV), torch.empty_like(q))
    x = v_new.float() / torch.tensor(scales, dtype=torch.float32).reshape(-1, 1)
    want = torch.where(x.isnan(), x, x.clamp(-448, 448)).to(torch.float8_e4m3fn).transpose(1, 2).reshape(n_rows, 128)
    nan = want.float().isnan()
    for got in (k.cpu(), v.cpu()):
        assert torch.equal(got.view(torch.float8_e4m3fn).float().isnan(), nan)
        assert torch.equal(got[~nan], want.view(torch.uint8)[~nan])


@pytest.mark.parametrize("page", [0, 16])
def test_accept_of_nothing_leaves_the_smallest_lengths_alone(page):
    """The draft's rows cannot be taken from a length of -2^31: the difference is no number of 32 bits."""
    s = Setup([[20, 9]], 2, 64, page=page, seed=7)
    s.lens_h = np.array([[-2 ** 31, 9]])
    s.make()
    bad = I32([0])
    F.fairkv_accept(s.cache, s.lens, I32(np.zeros((1, 6))), I32([0]), bad=bad)
    assert s.lens.cpu().tolist() == [[-2 ** 31, 3]] and int(bad) == 1


@pytest.mark.parametrize("q_len", WIDTHS)
def test_scores_of_minus_infinity_count_as_rows_that_are_not_seen(q_len):
    s = Setup([[70, 70, 2], [300, 300, 300]], q_len, 64, seed=11)
    s.lens_h = s.lens_h + q_len
    s.make()
    q = torch.randn(2, q_len, 24, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    q[..., 0] = 1
    for p in range(6):
        rows = [s.row(p, t) for t in range(int(s.lens_h.reshape(-1)[p]))]
        s.k[rows if p != 1 else rows[1:], 0] = -math.inf         # pair 1: but for its first row
    got, lse = (x.cpu() for x in _attend(s, 24, q_len, torch.float32, n_slots=16, q=q)[1:3])
    first = s.v[s.row(1, 0)].float().cpu().expand(q_len, 8, 64)
    # a weight p next to 1 in three parts, (p v) (1 / p): three sums of the parts' products, a quotient and a product, 2^-24 each
    assert ((got[0, :, 8:16] - first).abs() <= 2.0 ** -21 * first.abs()).all() and lse[0, :, 8:16].isfinite().all()
    got[0, :, 8:16], lse[0, :, 8:16] = 0, -math.inf
    assert not got.any() and (lse == -math.inf).all()


def test_a_packed_run_that_sticks_out_of_the_cache():
    """It is not attended to; what accept moves lies inside, and so does not move where it would not; an append behind it is left alone."""
    s = Setup([[40, 40]], 8, 64, seed=12)
    s.off[0] = s.n_rows - 38                                     # tokens 38 and 39 have no row
    s.make()
    q, out, lse, _ = _attend(s, 2, 4, torch.float32, n_slots=4)
    assert not out[:, :, 0].any() and (lse[:, :, 0] == -math.inf).all() and lse[:, :, 1].isfinite().all()
    k0, v0 = s.k.clone(), s.v.clone()
    for path, moved in (([3, 1, 0, 0], False), ([1, 0, 0, 0], True)):
        s.k.copy_(k0), s.v.copy_(v0)
        bad, lens = I32([0]), torch.zeros_like(s.lens)
        F.fairkv_accept(s.cache, s.lens, I32([path]), I32([2]), lens_out=lens, bad=bad)
        assert lens.cpu().tolist() == [[38 if moved else 40, 38]] and int(bad) == (0 if moved else 1)
        ref_k, ref_v = k0.clone(), v0.clone()
        for p in range(0 if moved else 1, 2):
            at = [s.row(p, 36 + i) for i in range(2)], [s.row(p, 36 + i) for i in path[:2]]
            ref_k[at[0]], ref_v[at[0]] = k0[at[1]], v0[at[1]]
        assert torch.equal(s.k, ref_k) and torch.equal(s.v, ref_v)
    bad, rows = I32([0]), torch.ones(1, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    F.fairkv_append_rotated(s.cache, s.lens, rows, rows, rows, torch.empty_like(rows), bad=bad)
    assert s.lens.cpu().tolist() == [[40, 41]] and int(bad) == 1


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("kv8", 16)])
def test_one_token_without_its_dimension_and_words_without_a_sign(dtype, page):
    """[B, H, D] is [B, 1, H, D], pages [B * Hkv, n] are [B, Hkv, n], a uint64 word is an int64 one: the same bits."""
    s = Setup([[70, 9], [300, 0]], 4, 128, dtype, page, seed=14, scales=True)
    q, k_new, v_new = (torch.randn(2, 1, h, 128, generator=torch.Generator().manual_seed(h)).to(torch.bfloat16).to(DEV) for h in (16, 2, 3))
    v_new = v_new[:, :, 1:]
    k0, v0, results = s.k.clone(), s.v.clone(), []
    for flat in (False, True):
        s.k.copy_(k0), s.v.copy_(v0)
        pages = {} if not page else dict(pages=I32(s.pages.reshape(2, 2, -1) if flat else s.pages), page_rows=page)
        kw = dict(k_scale=s.ks.tolist(), v_scale=s.vs.tolist()) if dtype == "kv8" else {}
        cache = F.Cache(s.k, s.v, I32(s.cap_h), **kw, **(pages or dict(off=torch.as_tensor(s.off if flat else s.off.reshape(2, 2), device=DEV))))
        x = [t[:, 0] if flat else t for t in (q, k_new, v_new)]
        lens, q_out, lse = I32(s.lens_h), torch.empty_like(x[0]), torch.empty(x[0].shape[:-1], device=DEV)
        out = torch.empty(q_out.shape, device=DEV)
        F.fairkv_append_rotated(cache, lens, *x, q_out, q_norm=torch.ones(128, device=DEV))
        tree = torch.full((2, 1), 1, dtype=torch.uint64 if flat else torch.int64, device=DEV)
        F.fairkv_decode_attn_tree(cache, lens, q_out, torch.zeros(F.fairkv_tree_workspace_bytes(cache, 16, 1), dtype=torch.uint8, device=DEV), out, lse, 0.1, tree=tree)
        F.fairkv_accept(cache, lens, I32([[0], [0]]), I32([1, 0]))
        results.append([t.flatten() for t in (lens, q_out, out, lse, s.k.view(torch.uint8), s.v.view(torch.uint8))])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert results[0][0].tolist() == [71, 10, 300, 0] and results[0][2].isfinite().all()
