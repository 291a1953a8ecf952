"""ss_logit_rules where a row's blocks have several windows of its vocabulary each, and where a list is as long as its entries can be numbered."""
import numpy as np
import pytest
import torch

import test_gpu_logit_rules as rules
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("half,in_place", [(False, False), (True, True)])
@pytest.mark.parametrize("bias", [False, True])
def test_many_rows_with_long_lists(bias, half, in_place):
    """More rows than there is a block a window for (16 blocks an SM): 700 of four windows, or seven beside biases."""
    r = np.random.default_rng(41)
    n, v = 700, 40000
    lists = [rules.text(r, int(x), v) for x in r.integers(2700, 3300, 8)]
    lists = [[t * (1 + i % 3) % v for t in x] for i, x in enumerate(lists)]                # (all over the vocabulary, too)
    c = rules.Case(41, n, v, half, history=[lists[s % 8] if s % 5 else [s] for s in range(n)], prompts=[[int(x) for x in r.integers(0, v, 3000)], [5]],
                   prompt_of=[s % 3 - 1 for s in range(n)], r=1.2, f=0.1, p=0.3, in_place=in_place,
                   bias=[[(int(t), float(b)) for t, b in zip(r.integers(0, v, 400), r.normal(size=400))]] if bias else None, bias_of=[0] * n if bias else None)
    B.ss_logit_rules(c.rules)
    c.check()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("v", [100, 5000, 6144, 6145, 7000, 9924, 12288, 12289, 20000, 151936])
@pytest.mark.parametrize("kind", ["history", "prompts", "bias", "all"])
def test_tokens_behind_the_vocabulary_are_in_no_window(kind, v, half):
    """Lists too long for the hash table, with tokens that a whole window at the vocabulary's end would reach, and further ones.  Behind every row
    there is room for them, which is left alone."""
    r = np.random.default_rng(v)
    rows, room = 5, 20000
    tokens = [int(t) for t in np.concatenate([r.integers(max(0, v - 3000), v + 100, 2000), r.integers(v - 5, v + 13000, 2500), [-1, -2, -(1 << 31), (1 << 31) - 1]])]
    r.shuffle(tokens)
    kw = dict(r=1.2, f=0.5)
    if kind in ("history", "all"):
        kw["history"] = [tokens] * rows
    if kind in ("prompts", "all"):
        kw.update(prompts=[tokens], prompt_of=[0] * rows)
    if kind in ("bias", "all"):
        kw.update(bias=[[(t, float(b)) for t, b in zip(tokens, r.normal(size=len(tokens)))]], bias_of=[0] * rows)
    for in_place in (False, True):
        c = rules.Case(v, rows, v, half, in_place=in_place, stride=v + room, **kw)
        behind = c.out.as_strided((rows, room), (v + room, 1), v)
        before = behind.clone()
        B.ss_logit_rules(c.rules)
        c.check()
        assert torch.equal(behind, before)


def test_the_longest_list():
    """More entries than 32 bits number: it ends, and the first 2^31 - 2049 count."""
    n = (1 << 31) + 100
    history = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    counted = (1 << 31) - 2049
    for at, token in ((0, 3), (5, 7), (1 << 30, 7), (counted - 1, 9), (counted, 11), (n - 1, 13)):
        history[at] = token
    x = torch.zeros(1, 1000, device=DEV)
    B.ss_logit_rules(B.make_logit_rules(logits=x, history=history, history_offsets=torch.tensor([0, n], device=DEV), frequency=1.0))
    want = torch.zeros_like(x)
    want[0, 3], want[0, 7], want[0, 9] = -1, -2, -1
    assert torch.equal(x, want)
