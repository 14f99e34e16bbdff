"""Attention weights of a growing cache on the GPU where numbers are none: a node whose log-sum-exp is -inf sees nothing and gives no weight to any row."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2502_15804_amd as F
from test_gpu_step import DEV, I32, Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "kv8"])
@pytest.mark.parametrize("D,G,n", [(128, 4, 2), (64, 4, 2), (128, 3, 40), (64, 8, 30), (128, 8, 40), (64, 16, 64), (128, 16, 64)])
def test_nodes_that_see_nothing_give_no_weight_to_rows_of_any_value(dtype, D, G, n):
    """One sequence where some nodes see nothing, and one where none does; infinite rows and NaN ones that only the nodes of no weight could add to."""
    s = Setup([[n + 100, n + 33], [n + 70, n]], 3, D, dtype, page=16, seed=n)
    gen = torch.Generator().manual_seed(D + n)
    q = torch.randn(2, n, 2 * G, D, generator=gen).to(torch.bfloat16).to(DEV)
    lse = (4 + torch.rand(2, n, 2 * G, generator=gen)).to(DEV)
    old = torch.rand(s.n_rows, generator=gen).to(DEV)
    rows = lambda b: [s.row(2 * b + h, t) for h in range(2) for t in range(int(s.lens_h[b, h]))]
    run = lambda lse: (out := old.clone(), F.fairkv_attn_weights(s.cache, s.lens, q, lse, out, 0.1, decay=0.5))[0]

    # some of the nodes: finite rows have what they have from the others, whatever their queries are
    some = lse.clone()
    some[0, ::2] = -math.inf
    want = run(some)
    others = q.clone()
    others[0, ::2] = 3.0
    q, keep = others, q
    assert torch.equal(run(some), want) and bool(torch.isfinite(want).all())
    q = keep
    assert torch.equal(run(some)[rows(1)], run(lse)[rows(1)])
    # all of them, over rows of every kind: what was there, and 0 for the new tokens' own
    none = lse.clone()
    none[0] = -math.inf
    bits = s.k.view(torch.uint8)
    for h in range(2):
        length = int(s.lens_h[0, h])
        for i, t in enumerate((0, 5, 31, 32, length - n, length - 1)):
            row = s.row(h, t)
            if dtype == "kv8":
                bits[row] = 0x7f
            else:
                s.k[row] = (math.inf, -math.inf, math.nan)[i % 3]
    got = run(none)
    for h in range(2):
        length = int(s.lens_h[0, h])
        at = [s.row(h, t) for t in range(length)]
        assert torch.equal(got[at[:length - n]], 0.5 * old[at[:length - n]]) and bool((got[at[length - n:]] == 0).all())
    assert torch.equal(got[rows(1)], want[rows(1)])
    # one of them left: those rows are no numbers for it, and so they are again
    if dtype == "bf16":
        none[0, 0] = 4.0
        got = run(none)
        assert bool(torch.isnan(got[s.row(0, 31)])) and bool(torch.isfinite(got[s.row(0, 6)]))


def test_log_sum_exps_at_the_end_of_their_range():
    """The lowest finite one is a number: rows get more weight than fp32 holds."""
    s = Setup([[40]], 0, 64)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(s.n_rows, device=DEV)
    rows = [s.row(0, t) for t in range(40)]
    for value, want in ((-3.4e38, math.inf), (3.4e38, 0.0), (math.inf, 0.0), (-math.inf, 0.0)):
        F.fairkv_attn_weights(s.cache, s.lens, q, torch.full((1, 1), value, device=DEV), out, 0.1)
        assert bool((out[rows] == want).all()), value
