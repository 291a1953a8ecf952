"""ss_key_weights where its inputs are at their ends."""
import ctypes
import math

import pytest
import torch

import test_gpu_key_weights as weights
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
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


# ---- rows that add nothing, rows that are not finite -----------------------------------------------------
@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_rows_that_are_switched_off_may_hold_anything(value, flags):
    c = weights.Case(33, 12, 2, [[64, 200], [64, 9]], [40, 2], shared=(0,))
    c.lse[7], c.lse[41], c.lse[20, 4], c.lse[33, 9] = (-math.inf,) * 4
    c.q[7], c.q[41, :, 5], c.q[20, 4], c.q[33, 9, 17] = (value,) * 4
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("hq,hkv,T", [(12, 2, 40), (32, 8, 64), (128, 1, 3), (1, 1, 1)])
def test_where_every_row_is_switched_off_the_weights_are_zero(hq, hkv, T, flags):
    c = weights.Case(34, hq, hkv, [[64, 200], [64, 9]], [T, 2], shared=(0,), decay=0.0)
    c.lse.fill_(-math.inf)
    assert c.run(flags) == B.SS_OK
    written = c.expected()[3]
    assert (c.weights[written] == 0).all()
    c.check()


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("kind", ["nan", "inf", "lse nan", "lse inf", "lse far below"])
@pytest.mark.parametrize("column", [0, 3, 14, 15, 46, 47, 62, 79, 100, 110, 111, 119])
def test_a_row_that_is_not_finite(column, kind, flags):
    """One query row of a step (token column / 6, head column % 6 of the second group of 6): what exp(s - lse) comes to reaches the weights of
    the keys that it sees, whichever unit the exponential of its column is taken by, and no other."""
    c = weights.Case(35, 12, 2, [[64, 200], [64, 9]], [20, 2], shared=(0,))
    t, h = column // 6, 6 + column % 6
    lse = float(c.lse[t, h])
    c.lse[t, h] = -math.inf
    want, tol, _, written = c.expected()
    c.lse[t, h] = lse
    if kind == "nan":
        c.q[t, h, 9] = float("nan")
    elif kind == "inf":
        c.q[t, h, 9] = float("inf")
    else:
        c.lse[t, h] = {"lse nan": float("nan"), "lse inf": float("inf"), "lse far below": -3e38}[kind]
    s, vis, _ = c.scores(0)
    term = torch.where(vis[h, t], torch.exp(s[h, t] - c.lse[t, h].double()), 0)       # 0, inf or NaN
    term = torch.where(term > 3.5e38, math.inf, term)                                # (as fp32 holds it)
    assert not (torch.isfinite(term) & (term != 0)).any()
    at = 0
    for n in c.chain[0]:
        i = torch.arange(c.lens[n], device=DEV)
        want[c.pages.long()[c.off[n] + i // 16], 1, i % 16] += term[at:at + c.lens[n]]
        at += c.lens[n]
    assert c.run(flags) == B.SS_OK
    got, fin = c.weights.double(), torch.isfinite(want)
    assert torch.equal(torch.isnan(got)[written], torch.isnan(want)[written])
    assert torch.equal(torch.isposinf(got)[written], torch.isposinf(want)[written])
    assert ((got - want).abs() <= tol)[written & fin].all()


# ---- very many keys, very many rows ----------------------------------------------------------------------
def alike(hq, lens, parent, leaf, pages, q, lse):
    """A descriptor over a pool of one kv head and few pages, which nodes have many times over (a page's keys get the same weight wherever the
    page is, so it may be written any number of times)."""
    i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
    n = len(leaf) if isinstance(leaf, list) else leaf.numel()
    off = [0]
    for x in lens:
        off.append(off[-1] + -(-x // 16))
    pool = pages["pool"]
    keep = [torch.tensor(parent, **i32), torch.tensor(lens, **i32), torch.tensor(off, **i64), torch.as_tensor(leaf, **i32),
            torch.ones(n, **i32), torch.arange(n + 1, **i64), torch.zeros(n, **i64), pool, pages["of"], q, lse]
    d = B.make_attn_desc(
        num_q_heads=hq, num_kv_heads=1, k_pool=pool[:, 0], v_pool=pool[:, 1], num_pages=pool.shape[0], kv_page_stride=pool.stride(0),
        kv_head_stride=2048, kv_token_stride=128, node_parent=keep[0], node_kv_len=keep[1], node_page_offsets=keep[2], node_pages=pages["of"],
        total_node_pages=off[-1], path_leaf_node=keep[3], path_q_len=keep[4], q_offsets=keep[5], total_q=n, q=q, out=torch.empty(n, 1, 1, device=DEV),
        lse=lse, q_src_offsets=keep[6], q_src_rows=1)
    d._keep = keep                                                # (a descriptor holds addresses alone)
    return d


@pytest.mark.parametrize("hq,hidden", [(128, True), (128, False), (32, True)])
def test_keys_far_in_front_of_a_nodes_end(hq, hidden):
    """More than 2^31 / heads keys in front of it: 17 million of 128 heads, 67 million of 32.  hidden: the node is the step's own leaf."""
    g = torch.Generator(device=DEV).manual_seed(36)
    n = (1 << 31) // hq + 2048
    pool = torch.randn(2, 2, 1, 16, 128, generator=g, device=DEV).bfloat16()
    lens = [n] if hidden else [n, 1]
    of = torch.ones(sum(-(-x // 16) for x in lens), dtype=torch.int32, device=DEV)
    of[:64] = 0                                                   # (page 0 holds the first 1024 keys, page 1 all others)
    q = torch.randn(1, hq, 128, generator=g, device=DEV).bfloat16()
    lse = torch.full((1, hq), 3.0, device=DEV)
    d = alike(hq, lens, [-1] if hidden else [-1, 0], [0] if hidden else [1], dict(pool=pool, of=of), q, lse)
    w = torch.full((2, 1, 16), 7.0, device=DEV)
    kw = B.make_key_weights(weights_out=w)
    ws = B.alloc_workspace(B.ss_key_weights_workspace_bytes(d, kw), DEV)
    B.ss_key_weights(d, kw, ws)
    assert B.ss_last_device_status(ws) == B.SS_OK
    k, x = pool[:, 0, 0].double(), q[0].double()                 # [2][16][128], [hq][128]
    s, size = k @ x.T / math.sqrt(128), k.abs() @ x.abs().T / math.sqrt(128)
    e = torch.exp(s - 3)
    tol = (e * (130 * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs() + 3) + 2.0 ** -21)).sum(-1) + e.sum(-1) * 50 * 2.0 ** -24
    assert ((w[:, 0].double() - e.sum(-1)).abs() <= tol).all()


def test_a_unit_of_more_steps_than_a_wait_is_long():
    """260000 rows of 128 heads below 768 keys, on one SM: a pair of tiles takes a step for each of them, some 0.3 s, and the warps that load
    the keys behind the next pair wait for all of it."""
    g = torch.Generator(device=DEV).manual_seed(37)
    hq, n = 128, 260000
    pool = torch.randn(48, 2, 1, 16, 128, generator=g, device=DEV).bfloat16()
    q = torch.randn(1, hq, 128, generator=g, device=DEV).bfloat16()
    lse = torch.full((n, hq), 3.0, device=DEV)
    d = alike(hq, [768], [-1], torch.zeros(n, dtype=torch.int32), dict(pool=pool, of=torch.arange(48, dtype=torch.int32, device=DEV)), q, lse)
    d.max_sms = 1
    w = torch.full((48, 1, 16), 7.0, device=DEV)
    kw = B.make_key_weights(weights_out=w)
    ws = B.alloc_workspace(B.ss_key_weights_workspace_bytes(d, kw), DEV)
    B.ss_key_weights(d, kw, ws)
    assert B.ss_last_device_status(ws) == B.SS_OK
    k, x = pool[:, 0, 0].double(), q[0].double()
    s, size = k @ x.T / math.sqrt(128), k.abs() @ x.abs().T / math.sqrt(128)
    e = torch.exp(s - 3)
    # (the same in every step, and the steps' sums are added up one by one)
    off = (e * (130 * 2.0 ** -23 * size + 2.0 ** -22 * (s.abs() + 3) + 2.0 ** -21)).sum(-1) + e.sum(-1) * (50 + n) * 2.0 ** -24
    assert ((w[:, 0].double() / n - e.sum(-1)).abs() <= off).all()


# ---- SMs -------------------------------------------------------------------------------------------------
class KernelNode(ctypes.Structure):
    _fields_ = [("func", ctypes.c_void_p)] + [(x, ctypes.c_uint) for x in ("gx", "gy", "gz", "bx", "by", "bz", "shared")] + \
        [("params", ctypes.c_void_p), ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def grids(call):
    """Blocks of the kernels that `call` launches (captured, not run)."""
    cuda = ctypes.CDLL("libcuda.so.1")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, count = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert cuda.cuGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert cuda.cuGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    blocks = []
    for node in nodes:
        kind = ctypes.c_int(-1)
        assert cuda.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value == 0:                                       # a kernel
            k = KernelNode()
            assert cuda.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(k)) == 0
            blocks.append(k.gx * k.gy * k.gz)
    return blocks


@pytest.mark.parametrize("flags", PATHS)
@pytest.mark.parametrize("sms", [1, 6, 20])
def test_a_bound_on_the_sms_is_kept_to(sms, flags):
    """By every kernel of the call: blocks are spread over the SMs first, so there are no more of them than that."""
    c = weights.Case(38, 12, 2, [[512, 1 + p % 50] for p in range(1024)], [1 + (p % 7 == 0) for p in range(1024)], shared=(0,))
    c.desc.flags, c.desc.max_sms = flags, sms
    blocks = grids(lambda: B.ss_key_weights(c.desc, c.kw, c.ws))
    assert len(blocks) == 2 and max(blocks) <= sms, blocks
    c.weights.copy_(c.untouched)
    c.order.fill_(-7)
    assert c.run(flags) == B.SS_OK
    c.check()


@pytest.mark.parametrize("flags", PATHS)
def test_a_million_rows(flags):
    """Queries of zero, so that every term is exp(-lse): off by 2^-21 at most, and by 2^-22 of |lse|.  The plain form adds them up in 64 bits, the
    tensor-core form by 128 and then, in two groups of half of the steps each, step by step."""
    n, lse = 1 << 20, 0.1
    pool = torch.randn(4, 2, 1, 16, 128, device=DEV).bfloat16()
    d = alike(1, [64], [-1], torch.zeros(n, dtype=torch.int32), dict(pool=pool, of=torch.arange(4, dtype=torch.int32, device=DEV)),
              torch.zeros(1, 1, 128, dtype=torch.bfloat16, device=DEV), torch.full((n, 1), lse, device=DEV))
    d.flags = flags
    w = torch.full((4, 1, 16), 7.0, device=DEV)
    kw = B.make_key_weights(weights_out=w)
    ws = B.alloc_workspace(B.ss_key_weights_workspace_bytes(d, kw), DEV)
    B.ss_key_weights(d, kw, ws)
    assert B.ss_last_device_status(ws) == B.SS_OK
    want = n * math.exp(-float(torch.tensor(lse)))
    steps = 0 if flags else n // 128 // 2 + 48
    assert ((w.double() - want).abs() <= want * (2.0 ** -21 + 0.1 * 2.0 ** -22 + 2.0 ** -23 + steps * 2.0 ** -24)).all()
