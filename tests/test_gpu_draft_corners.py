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


@pytest.mark.parametrize("flags", draft.PATHS)
def test_calls_without_rows_report_what_is_wrong(flags):
    """total_q = 0: nothing is written, and the status is what it is for any other call."""
    for what, want in (("nothing", B.SS_OK), ("steps", B.SS_ERR_BAD_INPUT), ("drafts", B.SS_ERR_UNSUPPORTED), ("leaf", B.SS_ERR_BAD_INPUT),
                       ("length", B.SS_ERR_BAD_INPUT), ("depth", B.SS_ERR_UNSUPPORTED)):
        chains = [[16] * (B.SS_MAX_DEPTH + 1), [40]] if what == "depth" else [[100], [40]]
        c = draft.Case(13, 8, 2, chains, [0, 0])
        node_parent, node_len, path_leaf, path_T, offs, q_offs = c.tensors
        if what == "steps":
            path_T[1] = 3
        elif what == "drafts":
            path_T[0] = B.SS_MAX_DRAFT + 1
        elif what == "leaf":
            path_leaf[1] = 2
        elif what == "length":
            node_len[0] = 1000
        assert c.desc.total_q == 0
        c.desc.q = c.desc.out = None                                     # (not needed without rows)
        assert c.run(flags) == want, what
        assert bool((c.out == 7).all()) and bool((c.lse == 7).all())
    # (no paths at all)
    c.desc.num_paths = 0
    assert c.run(flags) == B.SS_OK


def test_thousands_of_paths():
    """More paths than threads of a block: their costs are summed by stretches.  Every sixteenth against the definition, all of them
    against the plain kernel (both within their tolerance of 2e-2)."""
    r = torch.Generator().manual_seed(2)
    n = 3100
    chains = [[32, int(x)] for x in torch.randint(0, 40, (n,), generator=r)]
    T = torch.randint(0, 4, (n,), generator=r).tolist()
    c = draft.Case(17, 4, 2, chains, T, shared=(0,))
    assert c.run(B.SS_FLAG_FORCE_GENERIC) == B.SS_OK
    plain = c.out.clone(), c.lse.clone()
    for sms in (0, 3):
        c.desc.max_sms = sms
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        assert c.run() == B.SS_OK
        assert float((c.out.float() - plain[0].float()).abs().max()) <= 4e-2 and float((c.lse - plain[1]).abs().max()) <= 2e-3
        for p in range(0, n, 16):
            if T[p]:
                o, l, to, tl = c.exact(p)
                rows = slice(c.rows[p], c.rows[p] + T[p])
                assert bool(((c.out[rows].double() - o).abs() <= to).all()) and bool(((c.lse[rows].double() - l).abs() <= tl).all())
