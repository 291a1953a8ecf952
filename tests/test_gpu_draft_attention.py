"""ss_draft_attention against the definition in 64 bits.

Tolerance, element by element: the output's rounding to bf16 (2^-8 of it) and that of the probabilities (2^-8 of every term p_j v_j);
a score is a sum of 128 exact products in fp32, off by at most 130 * 2^-23 of scale * sum |q_d k_d| (the tensor cores cut off), a
logarithm-2 scaling by 2^-22 of itself, an exponential by 2^-22 - e(score) in all, which moves a term by that factor and the log-sum
by as much; another 2^-20 for the sums."""
import itertools
import math

import pytest
import torch

from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PATHS = [0, B.SS_FLAG_FORCE_GENERIC]


class Case:
    """Paths below a small tree.  chain[p]: node lengths root -> leaf in front of the drafts (the last gets T[p] drafts more); nodes
    with equal keys in `shared` are one node."""

    def __init__(self, seed, hq, hkv, chains, T, parents=None, shared=(), src=None, spread=1.0, pad_heads=0, dead=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.T, self.n = hq, hkv, T, len(T)
        lens, par, leaf, known, self.chain = [], [], [], {}, []
        for p, c in enumerate(chains):
            up, nodes = -1, []
            for i, x in enumerate(c):
                last = i == len(c) - 1
                key = (i, tuple(c[:i + 1])) if not last and i in shared else (p, i, "own")
                if key not in known:
                    known[key] = len(lens)
                    lens.append(x + (T[p] if last else 0))
                    par.append(up)
                up = known[key]
                nodes.append(up)
            leaf.append(up)
            self.chain.append(nodes)
        off = [0] + list(itertools.accumulate(-(-x // 16) for x in lens))
        rows = [0] + list(itertools.accumulate(T))
        self.lens, self.off, self.rows = lens, off, rows
        i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
        n_pages = off[-1] + 2
        self.pages = torch.randperm(n_pages, generator=g, device=DEV)[:max(off[-1], 1)].to(torch.int32)
        self.pool = torch.randn(n_pages, 2, hkv + pad_heads, 16, 128, generator=g, device=DEV).bfloat16()
        # slots behind a node's end, unused pages and padding heads hold NaN
        used = torch.zeros(n_pages, 16, dtype=torch.bool)
        for node, x in enumerate(lens):
            for t in range(x):
                used[int(self.pages[off[node] + t // 16]), t % 16] = True
        self.pool.masked_fill_(~used.to(DEV)[:, None, None, :, None], float("nan"))
        if pad_heads:
            self.pool[:, :, hkv:] = float("nan")
        self.src = rows[:-1] if src is None else src
        n_rows = rows[-1] if src is None else max(a + t for a, t in zip(src, T)) + 1
        self.q = (spread * torch.randn(n_rows, hq, 128, generator=g, device=DEV)).bfloat16()
        self.parent = torch.full((n_rows,), -7, **i32)
        self.parents = []
        for p, t in enumerate(T):
            one = parents[p] if parents else [int(torch.randint(-1, i, (1,), generator=r)) if i else -1 for i in range(t)]
            self.parents.append(one)
            if t:
                self.parent[self.src[p]:self.src[p] + t] = torch.tensor(one, **i32)
        self.out = torch.full((rows[-1] + 3, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((rows[-1] + 3, hq), 7.0, device=DEV)
        self.tensors = [torch.tensor(x, **i32) for x in (par, lens, leaf, T)] + [torch.tensor(off, **i64), torch.tensor(rows, **i64)]
        node_parent, node_len, path_leaf, path_T, offs, q_offs = self.tensors
        self.src_dev = torch.tensor(self.src, **i64)
        self.desc = B.make_attn_desc(
            num_q_heads=hq, num_kv_heads=hkv, k_pool=self.pool[:, 0], v_pool=self.pool[:, 1], num_pages=n_pages,
            kv_page_stride=self.pool.stride(0), kv_head_stride=2048, kv_token_stride=128, node_parent=node_parent, node_kv_len=node_len,
            node_page_offsets=offs, node_pages=self.pages, total_node_pages=off[-1], path_leaf_node=path_leaf, path_q_len=path_T,
            q_offsets=q_offs, total_q=rows[-1], q=self.q, out=self.out, lse=self.lse,
            q_src_offsets=None if src is None else self.src_dev, q_src_rows=0 if src is None else n_rows)
        self.ws = B.alloc_workspace(B.ss_draft_attention_workspace_bytes(self.desc), DEV)
        self.ws.fill_(0xEE)

    def run(self, flags=0, parent=True, **kw):
        self.desc.flags = flags
        B.ss_draft_attention(self.desc, self.parent if parent else None, self.ws, **kw)
        return B.ss_last_device_status(self.ws)

    def exact(self, p):
        """(out, lse, out tolerance, lse tolerance) of path p: [T][hq][128], [T][hq]."""
        T = self.T[p]
        kv = [torch.cat([self.pool[int(self.pages[self.off[n] + t // 16]), :, :self.hkv, t % 16][None] for n in self.chain[p]
                         for t in range(self.lens[n])] or [self.pool[:0, :, :self.hkv, 0]])[:, i].double() for i in (0, 1)]
        L = kv[0].shape[0]
        see = torch.zeros(T, T, dtype=torch.bool)
        for t in range(T):
            if self.parents[p][t] >= 0:
                see[t] = see[self.parents[p][t]]
            see[t, t] = True
        vis = torch.ones(T, L, dtype=torch.bool)
        for j in range(max(L - T, 0), L):
            vis[:, j] = see[:, j - (L - T)]
        vis = vis.to(DEV)
        outs, lses, to, tl = [], [], [], []
        rows = slice(self.src[p], self.src[p] + T)
        scale = 1 / math.sqrt(128)
        for h in range(self.hq):
            q, k, v = self.q[rows, h].double(), kv[0][:, h // (self.hq // self.hkv)], kv[1][:, h // (self.hq // self.hkv)]
            s = torch.where(vis, q @ torch.nan_to_num(k).T * scale, -math.inf)
            size = torch.where(vis, q.abs() @ torch.nan_to_num(k).abs().T * scale, 0)
            if L == 0:
                outs.append(torch.zeros(T, 128, dtype=torch.float64, device=DEV)); to.append(outs[-1])
                lses.append(torch.full((T,), -math.inf, dtype=torch.float64, device=DEV)); tl.append(torch.zeros_like(lses[-1]))
                continue
            lse = torch.logsumexp(s, 1)
            w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            v = torch.where(torch.isfinite(v), v, 0)
            o = w @ v
            e = (130 * 2.0 ** -23 * size.amax(1) + 2.0 ** -22 * torch.nan_to_num(s, neginf=0).abs().amax(1) + 2.0 ** -20)
            outs.append(o)
            lses.append(lse)
            to.append(2.0 ** -8 * o.abs() + (2.0 ** -8 + 2 * e)[:, None] * 1.01 * (w @ v.abs()) + 1e-30)
            tl.append(e + 2.0 ** -22 * torch.nan_to_num(lse, neginf=0).abs())
        return [torch.stack(x, 1) for x in (outs, lses, to, tl)]

    def check(self):
        for p in range(self.n):
            if self.T[p] == 0:
                continue
            o, l, to, tl = self.exact(p)
            rows = slice(self.rows[p], self.rows[p] + self.T[p])
            got, lse = self.out[rows].double(), self.lse[rows].double()
            assert bool(torch.isfinite(got).all()), p
            assert bool(((got - o).abs() <= to).all()), (p, float(((got - o).abs() - to).max()))
            fin = torch.isfinite(l)
            assert torch.equal(torch.isfinite(lse), fin) and bool((lse[~fin] == -math.inf).all())
            assert bool(((lse - l).abs()[fin] <= tl[fin]).all()), (p, float((lse - l).abs()[fin].max()))
        assert bool((self.out[self.rows[-1]:] == 7).all()) and bool((self.lse[self.rows[-1]:] == 7).all())


HEADS = [(12, 2), (28, 4), (8, 8), (16, 1), (128, 1), (40, 1)]


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("length", [0, 1, 15, 16, 100, 128, 257])
def test_one_path(flags, hq, hkv, length):
    for T in (1, 3, 17):
        c = Case(length + T, hq, hkv, [[length]], [T])
        assert c.run(flags) == B.SS_OK
        c.check()


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("hq,hkv", [(12, 2), (32, 8), (7, 1), (6, 6)])
def test_ragged_batch(flags, hq, hkv):
    """Paths of every kind in one call: long and short caches, chains with shared, empty and ragged inner nodes, no drafts, up to 128."""
    chains = [[300], [0], [64, 37], [64, 5], [32, 0, 16, 200], [1000], [21, 30], [5, 7, 9, 250], [2], [0, 0], [640], [16]]
    T = [7, 1, 30, 0, 64, 12, 128, 33, 65, 5, 1, 100]
    c = Case(hq, hq, hkv, chains, T, shared=(0,))
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
def test_tree_shapes(flags):
    """A chain, a star, a binary tree, all from the cached text, and the causal step without parents."""
    T = 70
    shapes = [[i - 1 for i in range(T)], [-1] + [0] * (T - 1), [(i - 1) // 2 if i else -1 for i in range(T)], [-1] * T]
    c = Case(3, 8, 2, [[50]] * 4, [T] * 4, parents=shapes)
    assert c.run(flags) == B.SS_OK
    c.check()
    c = Case(4, 8, 2, [[50], [3]], [T, 9], parents=[[i - 1 for i in range(T)], [i - 1 for i in range(9)]])
    assert c.run(flags, parent=False) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
def test_more_drafts_than_keys(flags):
    """A sequence that holds fewer tokens than there are drafts: rows that see nothing give 0 and -inf."""
    c = Case(5, 4, 2, [[-3], [-40], [-1]], [6, 41, 1])
    assert c.run(flags) == B.SS_OK
    c.check()
    assert bool((c.lse[0] == -math.inf).all()) and bool((c.out[0] == 0).all())


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_does_not_reach_it(flags, bad):
    """Keys and values of drafts outside a row's ancestors hold NaN or infinities; rows below them excepted, all is as without."""
    T = 40
    parents = [-1] + [0] * (T - 1)
    parents[20] = -1                                                     # nobody but itself sees draft 20
    c = Case(6, 12, 2, [[130], [700]], [T, T], parents=[parents, parents])
    for p in range(2):
        at = c.lens[c.chain[p][-1]] - T + 20
        page = int(c.pages[c.off[c.chain[p][-1]] + at // 16])
        c.pool[page, :, :, at % 16, 5:100] = bad
    keep = c.T
    assert c.run(flags) == B.SS_OK
    for p in range(2):
        o, l, to, tl = c.exact(p)
        rows = torch.tensor([r for r in range(T) if r != 20], device=DEV)
        got = c.out[c.rows[p] + rows].double()
        assert bool(torch.isfinite(got).all())
        assert bool(((got - o[rows]).abs() <= to[rows]).all())
        assert bool(((c.lse[c.rows[p] + rows].double() - l[rows]).abs() <= tl[rows]).all())
        assert not bool(torch.isfinite(c.out[c.rows[p] + 20].double()).all())
    assert c.T is keep


@pytest.mark.parametrize("flags", PATHS)
def test_scores_of_any_size(flags):
    """Scores in the hundreds (one key takes all) and next to nothing."""
    for spread in (60.0, 1e-3):
        c = Case(8, 8, 2, [[400], [90]], [20, 40], spread=spread)
        assert c.run(flags) == B.SS_OK
        c.check()


def _key(c, p, t, g):
    """Key row of token t of path p's own node."""
    n = c.chain[p][-1]
    return c.pool[int(c.pages[c.off[n] + t // 16]), 0, g, t % 16]


@pytest.mark.parametrize("sms", [0, 2])
@pytest.mark.parametrize("flags", PATHS)
def test_scores_that_rise_along_the_sequence(flags, sms):
    """A maximum that comes late: a little above what was before, far above, beyond what a float's exponent holds, again and again."""
    c = Case(30, 8, 2, [[900], [700], [260]], [50, 3, 64])
    c.desc.max_sms = sms
    for t, f in ((70, 6.0), (133, 30.0), (200, 400.0), (500, 1.5), (640, 900.0)):
        for g in range(2):
            _key(c, 0, t, g).mul_(f)
    for t in range(64, 700, 64):                                         # every half step above the last one
        for g in range(2):
            _key(c, 1, t, g).mul_(2.0 + t / 20)
    for t in range(1, 324):                                              # and a slope without an end
        _key(c, 2, t, 0).mul_(1 + t / 8)
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_cached_key_that_is_no_number(flags, what):
    """It is visible to every row of its head: none of them is finite, and the other head's are as they were."""
    c = Case(31, 8, 2, [[600]], [20])
    assert c.run(flags) == B.SS_OK
    before = c.out[:20].clone()
    _key(c, 0, 300, 0)[5] = what
    assert c.run(flags) == B.SS_OK
    finite = torch.isfinite(c.out[:20].double()).all(-1)
    if what != what:
        assert not bool(finite[:, :4].any())
    else:
        # a score of -inf has no weight, one of +inf leaves nothing else
        up = c.q[:20, :4, 5] > 0
        assert not bool(finite[:, :4][up].any()) and bool(finite[:, :4][c.q[:20, :4, 5] < 0].all())
    assert torch.equal(c.out[:20, 4:], before[:, 4:])


@pytest.mark.parametrize("flags", PATHS)
def test_query_rows_elsewhere_padded_pool_and_live_paths(flags):
    T = [5, 9, 33, 2]
    c = Case(9, 12, 2, [[100], [40], [333], [7]], T, src=[60, 3, 14, 50], pad_heads=1)
    live = torch.tensor([3], dtype=torch.int32, device=DEV)
    c.desc.num_paths_dev = live.data_ptr()
    assert c.run(flags) == B.SS_OK
    assert bool((c.out[c.rows[3]:] == 7).all())                          # the path that is not live
    c.T = T[:3] + [0]
    c.n, c.rows = 3, c.rows[:4]
    c.check()


@pytest.mark.parametrize("sms", [0, 1, 7])
def test_long_caches_over_few_and_many_blocks(sms):
    c = Case(10, 8, 2, [[5000], [9], [2100]], [16, 3, 40])
    c.desc.max_sms = sms
    assert c.run() == B.SS_OK
    c.check()
    again = c.out.clone(), c.lse.clone()
    for _ in range(3):                                                    # the same bits every time, whatever the workspace held
        c.ws.fill_(0x11)
        assert c.run() == B.SS_OK
        assert torch.equal(c.out, again[0]) and torch.equal(c.lse, again[1])


def test_many_paths():
    r = torch.Generator().manual_seed(1)
    n = 700
    chains = [[32, int(x)] for x in torch.randint(0, 60, (n,), generator=r)]
    T = torch.randint(0, 5, (n,), generator=r).tolist()
    c = Case(12, 4, 2, chains, T, shared=(0,))
    assert c.run() == B.SS_OK
    c.check()


def test_device_errors():
    for what in ("parent", "draft", "leaf", "page", "rows", "length"):
        c = Case(13, 8, 2, [[100], [40]], [5, 9])
        node_parent, node_len, path_leaf, path_T, offs, q_offs = c.tensors
        want = B.SS_ERR_BAD_INPUT
        if what == "parent":
            c.parent[3] = 3
        elif what == "draft":
            path_T[1] = 129
            want = B.SS_ERR_UNSUPPORTED
        elif what == "leaf":
            path_leaf[0] = 2
        elif what == "page":
            c.pages[1] = 1 << 20
        elif what == "rows":
            q_offs[1] = 10
        else:
            node_len[0] = 1000
        for flags in PATHS:
            assert c.run(flags) == want, what
        # the status is that of the last call
        d = Case(13, 8, 2, [[100], [40]], [5, 9])
        d.ws = c.ws
        assert d.run() == B.SS_OK
        d.check()


def test_graph_and_other_stream():
    c = Case(14, 12, 2, [[900], [40]], [16, 9])
    assert c.run() == B.SS_OK
    want = c.out.clone(), c.lse.clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.ss_draft_attention(c.desc, c.parent, c.ws)
    for _ in range(2):
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])
    # two calls at once, each with a workspace of its own
    d = Case(15, 12, 2, [[1500], [40]], [16, 9])
    torch.cuda.synchronize()
    for _ in range(5):
        B.ss_draft_attention(c.desc, c.parent, c.ws)
        B.ss_draft_attention(d.desc, d.parent, d.ws, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(c.out, want[0])
    d.check()


def test_causal_step_equals_the_tree_attention():
    """Without parents the call is ss_tree_attention on the same descriptor, within both accuracy contracts."""
    c = Case(16, 28, 4, [[64, 300], [64, 21]], [40, 17], shared=(0,), parents=[[i - 1 for i in range(40)], [i - 1 for i in range(17)]])
    assert c.run(parent=False) == B.SS_OK
    mine = c.out.clone(), c.lse.clone()
    ws = B.alloc_workspace(B.ss_tree_attention_workspace_bytes(c.desc), DEV)
    B.ss_tree_attention(c.desc, ws)
    assert B.ss_last_device_status(ws) == B.SS_OK
    assert float((mine[0].float() - c.out.float()).abs().max()) <= 2e-2 and float((mine[1] - c.lse).abs().max()) <= 1e-3
