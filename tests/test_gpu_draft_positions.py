"""Positions of drafts: draft t of a tree stands at the cached length plus its depth.  Index in the sequence - what ss_kv_append takes where
no positions are given - is that for a chain alone."""
import pytest
import torch

import test_gpu_draft_attention as draft
import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def appended(parents, positions, flags, same_rows):
    """A case of one path over 100 cached keys after ss_kv_append, and the drafts' keys in the pool."""
    T = len(parents)
    c = draft.Case(21, 12, 2, [[100]], [T], parents=[parents])
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v = rows_test.randn(g, T, 12, 128), rows_test.randn(g, T, 2, 128), rows_test.randn(g, T, 2, 128)
    if same_rows:
        for x in (q, k, v):
            x[:] = x[:1].clone()
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    B.ss_kv_append(c.desc, B.make_rows(q=q, k=k, v=v, q_out=c.q, positions=pos, inv_freq=rows_test.inv_freq(128)))
    assert c.run(flags) == B.SS_OK
    c.check()
    at = torch.arange(c.lens[0] - T, c.lens[0], device=DEV)
    return c, c.pool[c.pages.long()[at // 16], 0, :2, at % 16]


@pytest.mark.parametrize("flags", draft.PATHS)
def test_a_token_drafted_several_times_is_the_same_token(flags):
    parents = [-1, -1, -1, 0, 1, 3, 4]
    depth = [0, 0, 0, 1, 1, 2, 2]
    c, keys = appended(parents, [100 + d for d in depth], flags, same_rows=True)
    tol = c.exact(0)[2]
    for a in range(len(parents)):
        for b in range(a):
            if depth[a] == depth[b]:
                assert torch.equal(keys[a], keys[b])
                # the same keys and values, so the same exact rows, of which each is off by its tolerance at most
                assert bool(((c.out[a].double() - c.out[b].double()).abs() <= tol[a] + tol[b]).all())
    # by index in the sequence these are different tokens
    _, by_index = appended(parents, None, flags, same_rows=True)
    assert torch.equal(by_index[0], keys[0]) and not torch.equal(by_index[1], keys[1])


@pytest.mark.parametrize("flags", draft.PATHS)
def test_a_chain_needs_no_positions(flags):
    parents = [-1, 0, 1, 2, 3]
    a, keys = appended(parents, [100 + t for t in range(5)], flags, same_rows=False)
    b, by_index = appended(parents, None, flags, same_rows=False)
    assert torch.equal(keys, by_index) and torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
