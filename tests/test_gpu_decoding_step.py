"""The operators of a decoding step together, as a program runs them: the rows of a projection into the cache (ss_kv_append), a tree of
drafts over it (ss_draft_attention), the next tokens from the output layer's logits (ss_filtered_sample) - and with the deduplication in
front of them, whose arrays they take.  Each stage is compared in 64 bits on what the stage before it left."""
import pytest
import torch

import test_gpu_draft_attention as draft
import test_gpu_filtered_sample as sample
import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV, V = 12, 2, 5003


def make(seed, chains, T, **kw):
    """A draft case, the step's projected rows, and everything a program keeps for the step."""
    c = draft.Case(seed, HQ, HKV, chains, T, **kw)
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = c.q.shape[0]
    x = torch.randn(n, HQ + 2 * HKV, 128, generator=g, device=DEV).bfloat16()
    s = dict(c=c, x=x, q=x[:, :HQ], k=x[:, HQ:HQ + HKV], v=x[:, HQ + HKV:])
    s["wq"], s["wk"] = rows_test.weights(True, g)
    s["inv_freq"] = rows_test.inv_freq(128)
    depth = []
    for one in c.parents:
        d = []
        for up in one:
            d.append(d[up] + 1 if up >= 0 else 0)
        depth.append(d)
    pos = torch.zeros(n, dtype=torch.int32)
    for p, t in enumerate(T):
        cached = sum(c.lens[i] for i in c.chain[p]) - t
        pos[c.src[p]:c.src[p] + t] = cached + torch.tensor(depth[p], dtype=torch.int32) if t else pos[:0]
    s["positions"] = pos.to(DEV)
    s["rows"] = B.make_rows(q=s["q"], k=s["k"], v=s["v"], q_out=c.q, positions=s["positions"], inv_freq=s["inv_freq"], q_weight=s["wq"],
                            k_weight=s["wk"])
    total = c.rows[-1]
    s["head"] = (torch.randn(HQ * 128, V, generator=g, device=DEV) * 0.2).bfloat16()
    s["logits"] = torch.empty(total, V, dtype=torch.bfloat16, device=DEV)
    s["u"] = torch.rand(2 * total, generator=g, device=DEV)
    s["tokens"] = torch.full((2 * total,), -7, dtype=torch.int32, device=DEV)
    s["kept"] = torch.full((total,), -7, dtype=torch.int32, device=DEV)
    s["draws"] = torch.arange(0, 2 * total + 1, 2, dtype=torch.int64, device=DEV)
    s["sample"] = B.make_sample_desc(logits=s["logits"], draw_offsets=s["draws"], uniforms=s["u"], tokens_out=s["tokens"], kept_out=s["kept"],
                                     temperature=0.7, top_k=40, top_p=0.9)
    s["sample_ws"] = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(s["sample"]), DEV)
    return s


def step(s):
    c = s["c"]
    B.ss_kv_append(c.desc, s["rows"])
    B.ss_draft_attention(c.desc, c.parent, c.ws)
    torch.matmul(c.out[:c.rows[-1]].view(c.rows[-1], -1), s["head"], out=s["logits"])
    B.ss_filtered_sample(s["sample"], s["sample_ws"])


def verify(s):
    c = s["c"]
    assert B.ss_last_device_status(c.ws) == B.SS_OK
    for p, t in enumerate(c.T):
        if not t:
            continue
        r = torch.arange(c.src[p], c.src[p] + t, device=DEV)
        rows_test.close(c.q[r], *rows_test.turned(s["q"][r], s["wq"], s["positions"][r], s["inv_freq"], 128, False, 1e-6))
        leaf = c.chain[p][-1]
        at = torch.arange(c.lens[leaf] - t, c.lens[leaf], device=DEV)
        page = c.pages.long()[c.off[leaf] + at // 16]
        rows_test.close(c.pool[page, 0, :HKV, at % 16], *rows_test.turned(s["k"][r], s["wk"], s["positions"][r], s["inv_freq"], 128, False, 1e-6))
        assert torch.equal(c.pool[page, 1, :HKV, at % 16], s["v"][r])
    c.check()
    total = c.rows[-1]
    sums = s["tokens"].view(total, 2).cpu().numpy()
    x, u = s["logits"].double().cpu().numpy(), s["u"].view(total, 2).double().cpu().numpy()
    clear_rows = 0
    for i in range(total):
        ids, w, clear = sample.reference(x[i], 0.7, 40, 0.9, 0.0)
        if clear:
            clear_rows += 1
            assert int(s["kept"][i]) == len(ids)
            cum = w.cumsum()
            for j in range(2):
                if abs(cum - u[i, j] * cum[-1]).min() > sample.near(V) * cum[-1]:
                    assert sums[i, j] == ids[(cum <= u[i, j] * cum[-1]).sum()]
    assert clear_rows >= total - total // 8


def test_a_step_and_the_next_ones_in_a_graph():
    s = make(1, [[64, 200], [64, 37], [500], [7]], [16, 5, 33, 1], shared=(0,))
    step(s)
    verify(s)
    # captured once, replayed on new rows in the same buffers
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(s)
    for seed in (2, 3):
        g = torch.Generator(device=DEV).manual_seed(seed)
        s["x"].copy_(torch.randn(s["x"].shape, generator=g, device=DEV).bfloat16())
        s["u"].copy_(torch.rand(s["u"].shape, generator=g, device=DEV))
        graph.replay()
        verify(s)


def test_a_step_of_the_unique_paths():
    """Duplicates first: ss_dedup_paths and ss_gather_unique_paths on the device, then appending and attention for the unique paths,
    the rows read where they are."""
    s = make(5, [[40], [100], [40], [64, 9], [100]], [6, 9, 6, 20, 9], shared=(0,))
    c = s["c"]
    n = 5
    i32 = dict(dtype=torch.int32, device=DEV)
    same = [0, 1, 0, 3, 1]                                               # paths 2 and 4 repeat 0 and 1
    tok = torch.tensor(same, **i32)
    off = torch.arange(n + 1, dtype=torch.int64, device=DEV)
    outs = [torch.empty(n, **i32) for _ in range(4)]
    count = torch.zeros(1, **i32)
    B.ss_dedup_paths(tok, off, None, None, n, 0, outs[0], outs[1], outs[2], outs[3], None, count, B.alloc_workspace(B.ss_dedup_workspace_bytes(n), DEV))
    node_parent, node_len, path_leaf, path_T, offs, q_offs = c.tensors
    u_leaf, u_T = torch.empty(n, **i32), torch.empty(n, **i32)
    u_off, u_src = torch.empty(n + 1, dtype=torch.int64, device=DEV), torch.empty(n, dtype=torch.int64, device=DEV)
    B.ss_gather_unique_paths(outs[2], count, n, path_leaf, path_T, q_offs, u_leaf, u_T, u_off, u_src)
    d = c.desc
    d.path_leaf_node, d.path_q_len, d.q_offsets, d.q_src_offsets = u_leaf.data_ptr(), u_T.data_ptr(), u_off.data_ptr(), u_src.data_ptr()
    d.q_src_rows, d.num_paths_dev = c.rows[-1], count.data_ptr()
    before = c.pool.clone()
    c.ws = B.alloc_workspace(B.ss_draft_attention_workspace_bytes(d), DEV)
    B.ss_kv_append(d, s["rows"])
    B.ss_draft_attention(d, c.parent, c.ws)
    assert B.ss_last_device_status(c.ws) == B.SS_OK
    unique = [0, 1, 3]
    assert int(count) == 3 and outs[2][:3].tolist() == unique
    row = 0
    for p in unique:
        o, l, to, tl = c.exact(p)
        t = c.T[p]
        got, lse = c.out[row:row + t].double(), c.lse[row:row + t].double()
        assert bool(((got - o).abs() <= to).all()) and bool(((lse - l).abs() <= tl).all())
        row += t
    assert bool((c.out[row:] == 7).all())
    for p in (2, 4):                                                      # duplicates: nothing appended, queries left alone
        leaf = c.chain[p][-1]
        pages = c.pages[c.off[leaf]:c.off[leaf + 1]].long()
        assert torch.equal(torch.nan_to_num(c.pool[pages].float()), torch.nan_to_num(before[pages].float()))
