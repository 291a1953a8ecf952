"""ss_kv_evict against the definition, key by key on the host: everything that it leaves is a copy, so results are equal bit for bit."""
import itertools

import numpy as np
import pytest
import torch

from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


def reference(w, order, keep, sinks, recent):
    """Which slot's key every slot < k holds afterwards."""
    n = len(w)
    k = min(max(keep, 0), n)
    o = order.astype(np.int64)
    must = (o < sinks) | (o > (o.max() if n else 0) - recent)
    value = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
    # must stay first, then by weight with NaN behind -inf, then by slot
    ranked = sorted(range(n), key=lambda i: (not must[i], 0 if must[i] else np.isnan(w[i]), 0 if must[i] else -value[i], i))
    stay = np.sort(np.array(ranked[:k], dtype=np.int64))
    src = np.arange(k)
    free = np.setdiff1d(np.arange(k), stay)
    src[free] = stay[stay >= k]
    return src


class Case:
    def __init__(self, seed, lens, keep, hkv=2, listed=None, weights="rand", order=None, sinks=0, recent=0, separate=False, pad=0, max_keys=0,
                 alias_len=False):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.keep, self.hkv, self.sinks, self.recent = lens, keep, hkv, sinks, recent
        self.listed = list(range(len(lens))) if listed is None else listed
        self.off = [0] + list(itertools.accumulate(-(-x // 16) for x in lens))
        n_pages = self.off[-1] + 3
        self.pages = torch.randperm(n_pages, generator=g, device=DEV)[:max(1, self.off[-1])].to(torch.int32)
        self.pool = torch.randn(n_pages, 2, hkv + pad, 16, 128, generator=g, device=DEV).bfloat16()
        shape = (n_pages, hkv, 16)
        w = torch.rand(shape, generator=g, device=DEV)
        if weights == "ties":
            w = (w * 4).floor()
        elif weights == "equal":
            w.fill_(0.25)
        elif weights == "odd":
            bits = torch.randint(-(1 << 31), 1 << 31, shape, generator=g, device=DEV, dtype=torch.int64)
            w = bits.to(torch.int32).view(torch.float32)
            w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.2, float("nan"), w)
            w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, float("-inf"), w)
            w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, float("inf"), w)
            w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, -0.0, torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, 0.0, w))
        elif weights == "spread":
            w = torch.exp(20 * (w - 0.5))
        self.w = w.contiguous()
        self.order = None
        if order:
            self.order = torch.randint(0, 3 * max(lens) + 1, shape, generator=g, **I32)
        self.w_out = torch.full(shape, 7.0, device=DEV) if separate else None
        self.o_out = torch.full(shape, -7, **I32) if separate else None
        self.src = torch.full(shape, -7, **I32)
        self.len_dev = torch.tensor(lens, **I32)
        self.len_out = self.len_dev if alias_len else torch.full((len(lens),), -7, **I32)
        self.off_dev = torch.tensor(self.off, dtype=torch.int64, device=DEV)
        none32, none64 = torch.zeros(1, **I32), torch.zeros(2, dtype=torch.int64, device=DEV)
        self.desc = B.make_attn_desc(
            num_q_heads=hkv, num_kv_heads=hkv, k_pool=self.pool[:, 0], v_pool=self.pool[:, 1], num_pages=n_pages,
            kv_page_stride=self.pool.stride(0), kv_head_stride=2048, kv_token_stride=128, node_parent=torch.full((len(lens),), -1, **I32),
            node_kv_len=self.len_dev, node_page_offsets=self.off_dev, node_pages=self.pages, total_node_pages=self.off[-1], path_leaf_node=none32,
            path_q_len=none32, q_offsets=none64, total_q=0, q=None, out=None)
        self.nodes, self.keep_dev = torch.tensor(self.listed, **I32), torch.tensor([keep[x] for x in range(len(self.listed))], **I32)
        self.ev = B.make_evict(nodes=self.nodes, keep=self.keep_dev, weights=self.w, weights_out=self.w_out, order=self.order, order_out=self.o_out,
                               source_out=self.src, kv_len_out=self.len_out, sinks=sinks, recent=recent, max_keys=max_keys)
        self.ws = B.alloc_workspace(B.ss_kv_evict_workspace_bytes(self.desc, self.ev), DEV)
        self.ws.fill_(0xEE)
        self.expect()

    def expect(self):
        w, pages = self.w.cpu().numpy(), self.pages.cpu().numpy()
        order = None if self.order is None else self.order.cpu().numpy()
        self.want_pool = self.pool.clone()
        # (bit patterns, so that NaN compares)
        wb = self.w.view(torch.int32)
        self.want_w = (wb if self.w_out is None else self.w_out.view(torch.int32)).clone()
        self.want_o = None if self.order is None and self.o_out is None else (self.order if self.o_out is None else self.o_out).clone()
        self.want_src, self.want_len = self.src.clone(), self.len_out.clone()
        for x, node in enumerate(self.listed):
            n = self.lens[node]
            k = min(max(self.keep[x], 0), n)
            self.want_len[node] = k
            mine = pages[self.off[node]:self.off[node + 1]]
            place = lambda i: (torch.tensor(mine[i // 16], device=DEV).long(), torch.tensor(i % 16, device=DEV).long())  # noqa: E731
            for h in range(self.hkv):
                o = np.arange(n) if order is None else order[mine, h].reshape(-1)[:n]
                src = reference(w[mine, h].reshape(-1)[:n], o, self.keep[x], self.sinks, self.recent)
                to, of = place(np.arange(k)), place(src)
                self.want_pool[to[0], :, h, to[1]] = self.pool[of[0], :, h, of[1]]
                self.want_w[to[0], h, to[1]] = wb[of[0], h, of[1]]
                self.want_src[to[0], h, to[1]] = torch.tensor(src, **I32)
                if self.want_o is not None:
                    self.want_o[to[0], h, to[1]] = torch.tensor(o[src], **I32)

    def run(self, **kw):
        B.ss_kv_evict(self.desc, self.ev, self.ws, **kw)
        return B.ss_last_device_status(self.ws)

    def check(self):
        assert torch.equal(self.pool.view(torch.int16), self.want_pool.view(torch.int16))
        assert torch.equal((self.w if self.w_out is None else self.w_out).view(torch.int32), self.want_w)
        assert torch.equal(self.src, self.want_src) and torch.equal(self.len_out, self.want_len)
        if self.want_o is not None:
            assert torch.equal(self.order if self.o_out is None else self.o_out, self.want_o)


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 100, 500, 511, 512, 513, 1000]


@pytest.mark.parametrize("weights", ["rand", "ties", "equal", "odd", "spread"])
@pytest.mark.parametrize("share", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_small_nodes(weights, share):
    c = Case(1, LENS, [int(x * share) for x in LENS], weights=weights)
    assert c.run() == B.SS_OK
    c.check()


@pytest.mark.parametrize("order", [False, True])
@pytest.mark.parametrize("sinks,recent", [(0, 10), (4, 0), (4, 10), (100, 100), (0, 1 << 30), (1 << 30, 0)])
def test_keys_that_must_stay(sinks, recent, order):
    c = Case(2, LENS, [x // 2 for x in LENS], sinks=sinks, recent=recent, order=order, weights="ties")
    assert c.run() == B.SS_OK
    c.check()


@pytest.mark.parametrize("order", [False, True])
def test_outputs_of_their_own_and_again(order):
    c = Case(3, LENS, [x // 3 for x in LENS], sinks=2, recent=5, order=order, separate=True)
    for _ in range(2):                                            # (the second time on the pool that the first left)
        assert c.run() == B.SS_OK
        c.check()


@pytest.mark.parametrize("n,keep", [(2047, 1000), (5000, 4999), (8193, 1), (20000, 7000), (70001, 35000), (140000, 139000)])
@pytest.mark.parametrize("weights", ["rand", "ties", "odd"])
def test_long_nodes(n, keep, weights):
    c = Case(4, [n, 40], [keep, 20], hkv=1, weights=weights, sinks=4, recent=100)
    assert c.run() == B.SS_OK
    c.check()


def test_longer_than_said():
    c = Case(5, [70000, 3000], [30000, 100], hkv=2, weights="ties", max_keys=100, order=True, recent=50)
    assert c.run() == B.SS_OK
    c.check()


def test_many_nodes_some_of_them_padding_heads_lengths_in_place():
    r = np.random.default_rng(6)
    lens = [int(x) for x in r.integers(0, 700, 300)]
    listed = [int(x) for x in r.permutation(300)[:200]]
    c = Case(6, lens, [int(x) for x in r.integers(-5, 600, 200)], hkv=3, listed=listed, pad=1, alias_len=True, recent=7, separate=True)
    assert c.run() == B.SS_OK
    c.check()


def test_next_eviction_goes_by_what_the_first_left():
    """Evict, append, evict: the arrays in place, order from the first to the last."""
    c = Case(7, [600], [300], weights="rand", recent=20, sinks=4, alias_len=True)
    c.order = torch.zeros(c.w.shape, **I32)
    t = torch.arange(600, device=DEV)
    page = c.pages.long()[t // 16]
    c.order[page, :, t % 16] = t.to(torch.int32)[:, None]
    c.ev = B.make_evict(nodes=c.nodes, keep=c.keep_dev, weights=c.w, order=c.order, source_out=c.src, kv_len_out=c.len_out, sinks=4, recent=20)
    c.expect()
    assert c.run() == B.SS_OK
    c.check()
    kept = c.order[c.pages.long()[:19], 0].flatten()[:300]
    assert {0, 1, 2, 3, *range(580, 600)} <= set(kept.tolist())
    # 50 tokens more
    t = torch.arange(300, 350, device=DEV)
    page = c.pages.long()[t // 16]
    c.order[page, :, t % 16] = (t + 300).to(torch.int32)[:, None]
    c.w[page, :, t % 16] = 0
    c.len_dev.fill_(350)
    c.lens = [350]
    c.expect()
    assert c.run() == B.SS_OK
    c.check()
    kept = c.order[c.pages.long()[:19], 1].flatten()[:300]
    assert {0, 1, 2, 3, *range(630, 650)} <= set(kept.tolist())


@pytest.mark.parametrize("what", ["node", "negative node", "twice", "length", "page"])
def test_errors_that_the_device_finds(what):
    c = Case(8, [100, 200, 300, 400], [50, 60, 70, 80])
    before = c.pool.clone()
    if what == "node":
        c.nodes[1] = 4
    elif what == "negative node":
        c.nodes[1] = -1
    elif what == "twice":
        c.nodes[1] = 0
    elif what == "length":
        c.len_dev[1] = 1 << 30
    else:
        c.pages[c.off[1]] = 1 << 25
    assert c.run() == B.SS_ERR_BAD_INPUT
    for node in (0, 2, 3):                                        # the others are cut
        mine = c.pages[c.off[node]:c.off[node + 1]].long()
        assert torch.equal(c.pool[mine], c.want_pool[mine])
    if what != "page":
        mine = c.pages[c.off[1]:c.off[2]].long()
        assert torch.equal(c.pool[mine], before[mine]) and int(c.len_out[1]) == -7


def test_nothing_to_do():
    c = Case(9, [100], [50])
    before = c.pool.clone()
    c.ev.n_nodes = 0
    assert c.run() == B.SS_OK
    assert torch.equal(c.pool, before)


def test_graph_and_another_stream():
    c = Case(10, [1000, 300], [500, 299], separate=True, recent=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.ss_kv_evict(c.desc, c.ev, c.ws)
    s.synchronize()
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.ss_kv_evict(c.desc, c.ev, c.ws)
    c.w_out.fill_(7.0)
    c.o_out.fill_(-7)
    g.replay()
    torch.cuda.synchronize()
    c.check()
