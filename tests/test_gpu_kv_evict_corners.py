"""ss_kv_evict and pages that are not in the pool."""
import pytest
import torch

import test_gpu_kv_evict as evict
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entry", [0, 5, 12])
@pytest.mark.parametrize("keep", [0, -3, 60, 200, 300])           # none, none, some, all
@pytest.mark.parametrize("value", [-1, -(1 << 31), None, 1 << 30])
def test_a_page_that_is_not_in_the_pool(value, keep, entry):
    c = evict.Case(21, [100, 200, 300], [50, keep, 70])
    before = c.pool.clone()
    bad = int(c.pages[c.off[1] + entry])
    c.pages[c.off[1] + entry] = c.pool.shape[0] if value is None else value
    assert c.run() == B.SS_ERR_BAD_INPUT
    for node in (0, 2):                                           # the others are cut, and the page that is out of reach stays
        mine = c.pages[c.off[node]:c.off[node + 1]].long()
        assert torch.equal(c.pool[mine], c.want_pool[mine])
    assert torch.equal(c.pool[bad], before[bad])
    assert c.len_out.tolist() == [50, min(max(keep, 0), 200), 70]
