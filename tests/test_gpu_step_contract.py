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
