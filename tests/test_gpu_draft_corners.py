"""ss_draft_attention where its kernels take unusual ways: rows that are computed again over a long cache, thousands of paths, calls
without rows."""
import math

import pytest
import torch

import test_gpu_draft_attention as draft
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rows_computed_again_over_a_long_cache():
    """A draft that most rows do not see holds NaN, behind 30000 cached keys, on one SM: the rows of a unit are computed again key by key,
    which takes longer than any other wait may.  The unit behind it waits for that all the same."""
    T, hidden = 128, 20
    c = draft.Case(6, 4, 1, [[30000]], [T], parents=[[-1] * T])
    at = c.lens[0] - T + hidden
    c.pool[int(c.pages[at // 16]), :, :, at % 16, 5:100] = math.nan
    c.desc.max_sms = 1
    assert c.run() == B.SS_OK
    o, l, to, tl = c.exact(0)
    rows = torch.tensor([r for r in range(T) if r != hidden], device=DEV)
    got = c.out[rows].double()
    assert bool(torch.isfinite(got).all())
    assert bool(((got - o[rows]).abs() <= to[rows]).all()) and bool(((c.lse[rows].double() - l[rows]).abs() <= tl[rows]).all())
    assert bool(torch.isnan(c.out[hidden].double()).any(-1).all())
