"""ss_key_weights where its inputs are at their ends."""
import pytest
import torch

import test_gpu_key_weights as weights
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
PATHS = [0, B.SS_FLAG_FORCE_GENERIC]


# ---- pages -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("entry", [0, 7, 8, 17, 18])              # of a node of 300 keys: either tile of its first pair, the tile behind them
@pytest.mark.parametrize("value", [-1, -2, -(1 << 31), None, 1 << 30])
def test_a_page_that_is_not_in_the_pool(value, entry, flags):
    """It is reported whatever the entry says (-1 is how a page that is not there is mostly marked), and the other nodes' keys are right."""
    c = weights.Case(31, 12, 2, [[64, 20], [64, 291], [64, 9]], [4, 9, 1], shared=(0,))
    want, tol, order, written = c.expected()
    node = c.chain[1][-1]
    assert c.lens[node] == 300
    others = written.clone()
    others[c.pages[c.off[node]:c.off[node + 1]].long()] = False
    c.pages[c.off[node] + entry] = c.pool.shape[0] if value is None else value
    assert c.run(flags) == B.SS_ERR_BAD_INPUT
    assert ((c.weights.double() - want).abs() <= tol)[others].all()
    assert torch.equal(c.order.long()[others], order[others])
    assert torch.equal(c.weights[~written], c.untouched[~written])


@pytest.mark.parametrize("flags", PATHS)
def test_entries_behind_a_nodes_keys_may_hold_anything(flags):
    c = weights.Case(32, 12, 2, [[64, 20], [64, 291], [64, 9]], [4, 9, 1], shared=(0,))
    node = c.chain[1][-1]
    c.lens[node] = 250
    c.tensors[1][node] = 250
    for entry, value in ((16, -1), (17, -(1 << 31)), (18, 1 << 30)):
        spare = int(c.pages[c.off[node] + entry])
        c.pages[c.off[node] + entry] = value
        c.pool[spare] = float("nan")
    assert c.run(flags) == B.SS_OK
    c.check()
