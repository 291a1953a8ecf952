"""ss_key_weights against the definition in 64 bits, on the trees of the draft attention's tests.

Tolerance of a key's weight: of every term p = exp(s - lse), s is a sum of 128 exact products in fp32, off by at most 130 * 2^-23 of
scale * sum |q_d k_d| (the tensor cores cut off); scaled and the log-sum taken off it is off by 2^-23 of |s| and of |lse| each, rounded at
most twice; the power of two by 2^-21.  The sum of n terms: at most 48 additions deep and one for every 128 terms, 2^-24 each.  Then the
older weight and one rounding."""
import math

import pytest
import torch

import test_gpu_draft_attention as draft
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PATHS = [0, B.SS_FLAG_FORCE_GENERIC]


class Case(draft.Case):
    """The draft tests' tree with causal steps: their log-sums, weights and sequence numbers beside the pool."""

    def __init__(self, seed, hq, hkv, chains, T, last=0, decay=0.75, weights_in=True, path_order=True, in_place=False, **kw):
        super().__init__(seed, hq, hkv, chains, T, parents=[list(range(-1, t - 1)) for t in T], **kw)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        self.last, self.decay = last, decay
        shape = (self.pool.shape[0], hkv, 16)
        self.weights_in = torch.rand(shape, generator=g, device=DEV) if weights_in else None
        if decay == 0 and weights_in:
            self.weights_in.fill_(float("nan"))                   # (not read)
        self.before = self.weights_in.clone() if weights_in else torch.zeros(shape, device=DEV)
        self.weights = self.weights_in if in_place else torch.full(shape, 7.0, device=DEV)
        self.untouched = self.weights.clone()
        self.order = torch.full(shape, -7, dtype=torch.int32, device=DEV)
        self.path_order = torch.randint(0, 1 << 30, (max(len(T), 1),), generator=g, device=DEV, dtype=torch.int32) if path_order else None
        self.kw = B.make_key_weights(weights_out=self.weights, weights_in=self.weights_in, decay=decay, order=self.order,
                                     path_order=self.path_order, last_tokens=last)
        self.lse.fill_(float("nan"))
        for p in range(len(T)):
            s, vis, _ = self.scores(p)
            self.lse[self.rows[p]:self.rows[p] + T[p]] = torch.logsumexp(torch.where(vis, s, -math.inf), -1).T.float() if s.shape[-1] else -math.inf
        self.ws = B.alloc_workspace(B.ss_key_weights_workspace_bytes(self.desc, self.kw), DEV)
        self.ws.fill_(0xEE)

    def keys(self, node):
        """[hkv][keys][128] of a node."""
        t = torch.arange(self.lens[node], device=DEV)
        return self.pool[self.pages.long()[self.off[node] + t // 16], 0, :, t % 16][:, :self.hkv].transpose(0, 1).double()

    def scores(self, p):
        """Scores of path p, which of them a token sees, and their size: [hq][T][L]."""
        T, rep = self.T[p], self.hq // self.hkv
        k = torch.cat([self.keys(n) for n in self.chain[p]], 1).repeat_interleave(rep, 0)
        q = self.q[self.src[p]:self.src[p] + T].double().transpose(0, 1)
        L = k.shape[1]
        vis = (torch.arange(L, device=DEV)[None, :] <= L - T + torch.arange(T, device=DEV)[:, None])[None].expand(self.hq, T, L)
        k0 = torch.nan_to_num(k)
        scale = 1 / math.sqrt(128)
        return q @ k0.transpose(1, 2) * scale, vis, q.abs() @ k0.abs().transpose(1, 2) * scale

    def run(self, flags=0, **kw):
        self.desc.flags = flags
        B.ss_key_weights(self.desc, self.kw, self.ws, **kw)
        return B.ss_last_device_status(self.ws)

    def expected(self):
        """weights, tolerance, order, and which keys are written, beside the pool."""
        shape = self.before.shape
        want, tol = torch.zeros(shape, dtype=torch.float64, device=DEV), torch.zeros(shape, dtype=torch.float64, device=DEV)
        terms = torch.zeros(shape, dtype=torch.float64, device=DEV)
        new = torch.zeros(shape, dtype=torch.bool, device=DEV)
        written, order = torch.zeros_like(new), torch.full(shape, -7, dtype=torch.int64, device=DEV)
        for p, T in enumerate(self.T):
            if len(self.chain[p]) == 0:
                continue
            s, vis, size = self.scores(p)
            L = s.shape[-1]
            lse = self.lse[self.rows[p]:self.rows[p] + T].double().T[:, :, None]
            used = min(T, self.last) if self.last else T
            counts = vis & (torch.arange(T, device=DEV) >= T - used)[None, :, None] & (lse > -math.inf)
            e = torch.where(counts, torch.exp(s - lse), 0)
            off = torch.where(counts, e * (130 * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs() + lse.abs()) + 2.0 ** -21), 0)
            per_head = lambda x: x.sum(1).view(self.hkv, -1, L).sum(1)  # noqa: E731
            at = 0
            for n in self.chain[p]:
                i = torch.arange(self.lens[n], device=DEV)
                page, slot = self.pages.long()[self.off[n] + i // 16], i % 16
                cut = slice(at, at + self.lens[n])
                want[page, :, slot] += per_head(e)[:, cut].T
                tol[page, :, slot] += per_head(off)[:, cut].T
                terms[page, :, slot] += per_head(counts.double())[:, cut].T
                written[page, :, slot] = True
                at += self.lens[n]
            i = torch.arange(self.lens[n] - T, self.lens[n], device=DEV)
            page, slot = self.pages.long()[self.off[n] + i // 16], i % 16
            new[page, :, slot] = True
            first = int(self.path_order[p]) if self.path_order is not None else L - T
            order[page, :, slot] = (first + torch.arange(T, device=DEV))[:, None]
        tol += want * (48 + terms / 128) * 2.0 ** -24
        if self.decay:
            old = torch.where(new, 0, self.before.double() * self.decay)
            want += old
        return want, tol + want.abs() * 2.0 ** -23, order, written

    def check(self):
        want, tol, order, written = self.expected()
        got = self.weights.double()
        off = (got - want).abs()
        bad = written & ~(off <= tol)
        assert not bad.any(), (int(bad.sum()), int(written.sum()), float((off / tol)[written].nan_to_num(1e30).max()), bad.nonzero()[:5].tolist())
        assert torch.equal(self.order.long(), order)
        assert torch.equal(self.weights[~written], self.untouched[~written])


CASES = {
    "one token": dict(hq=1, hkv=1, chains=[[0]], T=[1]),
    "two keys": dict(hq=12, hkv=2, chains=[[1]], T=[1]),
    "tile ends": dict(hq=8, hkv=1, chains=[[126], [127], [128], [129], [255], [256]], T=[1] * 6),
    "steps over pages": dict(hq=12, hkv=2, chains=[[16, 100], [16, 7]], T=[37, 20], shared=(0,)),
    "more than a step of rows": dict(hq=28, hkv=4, chains=[[256, 40], [256, 90], [256, 1], [256, 130]], T=[40, 64, 1, 127], shared=(0,)),
    "deep": dict(hq=32, hkv=8, chains=[[33, 0, 17, 5], [33, 0, 17, 60], [33, 0, 48, 9], [33, 64, 9]], T=[3, 1, 9, 16], shared=(0, 1, 2)),
    "no sharing": dict(hq=16, hkv=16, chains=[[300], [0], [77]], T=[5, 3, 1]),
    "a path without tokens": dict(hq=12, hkv=2, chains=[[64, 20], [64, 30]], T=[0, 2], shared=(0,)),
    "no tokens at all": dict(hq=12, hkv=2, chains=[[64, 20], [64, 30]], T=[0, 0], shared=(0,)),
    "window": dict(hq=28, hkv=4, chains=[[200, 500], [200, 3]], T=[150, 40], shared=(0,), last=32),
    "window of one": dict(hq=12, hkv=2, chains=[[500]], T=[300], last=1),
    "a wide group": dict(hq=64, hkv=1, chains=[[150, 9]], T=[5]),
    "widest group": dict(hq=128, hkv=1, chains=[[150, 9], [150, 20]], T=[2, 1], shared=(0,)),
    "odd group": dict(hq=21, hkv=3, chains=[[100, 9], [100, 11]], T=[31, 9], shared=(0,)),
    "many paths": dict(hq=12, hkv=2, chains=[[512, 30 + p % 50] for p in range(100)], T=[1 + (p % 7 == 0) for p in range(100)], shared=(0,)),
    "long step": dict(hq=12, hkv=2, chains=[[0, 0]], T=[700]),
    "rows elsewhere": dict(hq=12, hkv=2, chains=[[64, 20], [64, 30], [64, 9]], T=[4, 9, 1], shared=(0,), src=[11, 0, 30]),
    "padding heads in the pool": dict(hq=12, hkv=2, chains=[[64, 200]], T=[20], pad_heads=1),
    "spread scores": dict(hq=12, hkv=2, chains=[[64, 200]], T=[20], spread=8.0),
    "no older weights": dict(hq=12, hkv=2, chains=[[64, 200]], T=[20], weights_in=False),
    "older weights forgotten": dict(hq=12, hkv=2, chains=[[64, 200]], T=[20], decay=0.0),
    "in place": dict(hq=12, hkv=2, chains=[[64, 200], [64, 10]], T=[20, 3], shared=(0,), in_place=True),
    "numbers by place": dict(hq=12, hkv=2, chains=[[64, 200], [64, 10]], T=[20, 3], shared=(0,), path_order=False),
}


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("name", CASES)
def test_weights(name, flags):
    c = Case(5, **CASES[name])
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
def test_rows_that_add_nothing(flags):
    c = Case(6, 12, 2, [[64, 50], [64, 9]], [6, 2], shared=(0,))
    c.lse[1] = -math.inf
    c.lse[3, 4] = -math.inf
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
def test_a_hidden_key_that_is_not_finite(flags):
    """The step's last keys hold NaN: they reach neither the other keys' weights nor, where no counted row sees them, their own."""
    c = Case(7, 12, 2, [[64, 50]], [6])
    n = c.chain[0][-1]
    want = c.expected()
    for i, v in ((c.lens[n] - 1, float("nan")), (c.lens[n] - 2, float("inf"))):
        c.pool[int(c.pages[c.off[n] + i // 16]), 0, :, i % 16] = v
    assert c.run(flags) == B.SS_OK
    written = want[3].clone()
    for i in (c.lens[n] - 1, c.lens[n] - 2):
        written[int(c.pages[c.off[n] + i // 16]), :, i % 16] = False
    off = (c.weights.double() - want[0]).abs()
    assert (off <= want[1])[written].all()


def test_a_long_node_is_shared_by_blocks_and_the_result_does_not_depend_on_the_run():
    c = Case(8, 28, 4, [[4096, 60 + p] for p in range(24)], [40] * 24, shared=(0,))
    assert c.run() == B.SS_OK
    c.check()
    first = c.weights.clone()
    for _ in range(3):
        assert c.run() == B.SS_OK
        assert torch.equal(c.weights, first)
    c.desc.max_sms = 5
    assert c.run() == B.SS_OK
    c.check()


def test_few_keys_and_very_many_rows():
    """A unit's rows go to all blocks."""
    c = Case(9, 32, 4, [[48, 1] for _ in range(300)], [20] * 300, shared=(0,))
    assert c.run() == B.SS_OK
    c.check()


def test_live_paths_are_counted_on_the_device():
    c = Case(10, 12, 2, [[64, 20], [64, 30], [64, 9]], [4, 9, 1], shared=(0,))
    live = torch.tensor([2], dtype=torch.int32, device=DEV)
    c.desc.num_paths_dev = live.data_ptr()
    assert c.run() == B.SS_OK
    c.T, c.chain = c.T[:2], c.chain[:2]
    c.check()
    live.zero_()
    c.weights.copy_(c.untouched)
    c.order.fill_(-7)
    assert c.run() == B.SS_OK
    assert torch.equal(c.weights, c.untouched) and (c.order == -7).all()


def test_no_paths():
    c = Case(11, 12, 2, [[64, 20]], [4])
    c.desc.num_paths = 0
    assert c.run() == B.SS_OK
    assert torch.equal(c.weights, c.untouched)


def bad(change, **kw):
    c = Case(12, 12, 2, [[64, 20], [64, 30], [64, 9]], [4, 9, 1], shared=(0,), **kw)
    par, lens, leaf, T = c.tensors[:4]
    change(c, par, lens, leaf, T)
    return c


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("what,status", [
    ("leaf", B.SS_ERR_BAD_INPUT), ("parent", B.SS_ERR_BAD_INPUT), ("page", B.SS_ERR_BAD_INPUT), ("length", B.SS_ERR_BAD_INPUT),
    ("rows", B.SS_ERR_BAD_INPUT), ("long step", B.SS_ERR_UNSUPPORTED), ("shared leaf", B.SS_ERR_UNSUPPORTED), ("loop", B.SS_ERR_UNSUPPORTED),
    ("not contiguous", B.SS_ERR_BAD_INPUT)])
def test_errors_that_the_device_finds(what, status, flags):
    def change(c, par, lens, leaf, T):
        if what == "leaf":
            leaf[1] = 99
        elif what == "parent":
            par[c.chain[1][-1]] = 99
        elif what == "page":
            c.pages[c.off[c.chain[1][-1]]] = 1 << 20
        elif what == "length":
            lens[c.chain[1][-1]] = 1000
        elif what == "rows":
            c.tensors[5][2] = 1 << 20
        elif what == "long step":
            lens[c.chain[1][-1]] = 8
        elif what == "shared leaf":
            leaf[1] = leaf[0]
        elif what == "loop":
            par[0] = 0
        else:                                                    # the middle path belongs to another root
            par[c.chain[1][-1]] = -1
    c = bad(change)
    assert c.run(flags) == status
    c = Case(13, 12, 2, [[64, 20]], [4])                          # and the next call is fine
    assert c.run(flags) == B.SS_OK
    c.check()


def test_graph_and_another_stream():
    c = Case(14, 12, 2, [[64, 200], [64, 10]], [20, 3], shared=(0,))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.ss_key_weights(c.desc, c.kw, c.ws)
    s.synchronize()
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.ss_key_weights(c.desc, c.kw, c.ws)
    for _ in range(2):
        c.weights.copy_(c.untouched)
        c.order.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        c.check()
