"""Steps of a search with a bounded cache, as a program runs them: the step's rows into the cache at explicit positions on several axes
(ss_kv_append_axes), attention (ss_tree_attention), the weight that every key received (ss_key_weights), the least of them out of the leaves
(ss_kv_evict), a step over what is left; and the logits behind their rules into a draw (ss_logit_rules, ss_filtered_sample).  Each stage is compared
in 64 bits on what the stage before it left."""
import math

import numpy as np
import pytest
import torch

import test_gpu_axes as axes_test
import test_gpu_key_weights as weights_test
import test_gpu_kv_evict as evict_test
import test_gpu_logit_rules as rules_test
import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV = 12, 2
I32 = dict(dtype=torch.int32, device=DEV)


def attend(c):
    """The attention of the step into c.out and c.lse, compared with the definition over the pool (bf16 outputs: 2^-8 of the size of the terms)."""
    ws = B.alloc_workspace(B.ss_tree_attention_workspace_bytes(c.desc), DEV)
    B.ss_tree_attention(c.desc, ws)
    assert B.ss_last_device_status(ws) == B.SS_OK
    for p, t in enumerate(c.T):
        s, vis, size = c.scores(p)
        s = torch.where(vis, s, -math.inf)
        v = torch.cat([c.pool[c.pages.long()[c.off[n] + torch.arange(c.lens[n], device=DEV) // 16], 1, :, torch.arange(c.lens[n], device=DEV) % 16]
                       for n in c.chain[p]]).double().transpose(0, 1).repeat_interleave(HQ // HKV, 0)
        rows = slice(c.rows[p], c.rows[p] + t)
        lse = torch.logsumexp(s, -1)
        w = torch.exp(s - lse[..., None])
        off = (130 * 2.0 ** -23 * size + 2.0 ** -20).amax(-1)
        assert ((c.lse[rows].double().T - lse).abs() <= off + 2.0 ** -20 * (1 + lse.abs())).all()
        tol = (w @ v.abs()) * (2.0 ** -8 + 2 * off[..., None]) + 2.0 ** -8 * (w @ v).abs() + 1e-6
        assert ((c.out[rows].double().transpose(0, 1) - w @ v).abs() <= tol).all()


def test_steps_with_a_bounded_cache():
    c = weights_test.Case(21, HQ, HKV, [[64, 90], [64, 61], [64, 130]], [5, 1, 16], shared=(0,), decay=0.9, in_place=True)
    g = torch.Generator(device=DEV).manual_seed(22)
    # numbers of the older keys; the step's come from ss_key_weights
    c.order.zero_()
    for p in range(3):
        leaf = c.chain[p][-1]
        t = torch.arange(c.lens[leaf], device=DEV)
        c.order[c.pages.long()[c.off[leaf] + t // 16], :, t % 16] = t.to(torch.int32)[:, None]
        c.path_order[p] = c.lens[leaf] - c.T[p]
    f, (wq, wk) = rows_test.inv_freq(128), rows_test.weights(True, g)
    pair_axis = torch.arange(64, **I32) % 3
    keep = [40, 61, 100]
    for step in range(3):
        n = c.rows[-1]
        x = rows_test.randn(g, n, HQ + 2 * HKV, 128)
        positions = torch.randint(0, 5000, (3, n), generator=g, **I32)
        r = B.make_rows(q=x[:, :HQ], k=x[:, HQ:HQ + HKV], v=x[:, HQ + HKV:], q_out=c.q, inv_freq=f, q_weight=wq, k_weight=wk)
        B.ss_kv_append_axes(c.desc, r, B.make_axes(positions=positions, pair_axis=pair_axis))
        rows_test.close(c.q, *axes_test.turned(x[:, :HQ], wq, positions, pair_axis, f, 128, False, 1e-6))
        attend(c)
        c.before = c.weights.clone()
        old_order = c.order.clone()
        assert c.run() == B.SS_OK
        want, tol, order, written = c.expected()
        assert ((c.weights.double() - want).abs() <= tol)[written].all()
        assert torch.equal(c.order.long(), torch.where(order >= 0, order, old_order.long()))
        # the leaves back into their budgets
        leaves = [c.chain[p][-1] for p in range(3)]
        pool, w, o, src = c.pool.clone(), c.weights.clone(), c.order.clone(), torch.full_like(c.order, -7)
        node_len = c.tensors[1]
        ev = B.make_evict(nodes=torch.tensor(leaves, **I32), keep=torch.tensor(keep, **I32), weights=c.weights, order=c.order, source_out=src,
                          kv_len_out=node_len, sinks=2, recent=8, max_keys=max(c.lens))
        ws = B.alloc_workspace(B.ss_kv_evict_workspace_bytes(c.desc, ev), DEV)
        B.ss_kv_evict(c.desc, ev, ws)
        assert B.ss_last_device_status(ws) == B.SS_OK
        pages = c.pages.cpu().numpy()
        for leaf, k in zip(leaves, keep):
            mine = torch.tensor(pages[c.off[leaf]:c.off[leaf + 1]], device=DEV).long()
            flat = lambda a, h: a[mine, h].flatten()  # noqa: E731
            kk = min(k, c.lens[leaf])
            for h in range(HKV):
                want_src = evict_test.reference(flat(w, h)[:c.lens[leaf]].cpu().numpy(), flat(o, h)[:c.lens[leaf]].cpu().numpy(), k, 2, 8)
                assert flat(src, h)[:kk].tolist() == want_src.tolist()
                at = torch.tensor(want_src, device=DEV)
                kv = lambda a: a[mine][:, :, h].transpose(1, 2).reshape(-1, 2, 128)  # noqa: E731
                assert torch.equal(kv(c.pool)[:kk], kv(pool)[at]) and torch.equal(flat(c.order, h)[:kk], flat(o, h)[at])
            c.lens[leaf] = kk
        assert node_len.tolist() == c.lens
        # the next step: as many tokens again behind what is left
        room = [16 * (c.off[x + 1] - c.off[x]) for x in leaves]
        for p, leaf in enumerate(leaves):
            assert c.lens[leaf] + c.T[p] <= room[p]
            c.path_order[p] += c.T[p]
            c.lens[leaf] += c.T[p]
        node_len.copy_(torch.tensor(c.lens, **I32))


def test_rules_in_front_of_a_draw():
    c = rules_test.everything(23, 6, 4001, False)
    tokens, kept = torch.zeros(12, **I32), torch.zeros(6, **I32)
    u = torch.rand(12, device=DEV)
    d = B.make_sample_desc(logits=c.out, draw_offsets=torch.arange(0, 13, 2, dtype=torch.int64, device=DEV), uniforms=u, tokens_out=tokens, kept_out=kept,
                           temperature=0.8, top_k=20)
    ws = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV)
    B.ss_logit_rules(c.rules)
    B.ss_filtered_sample(d, ws)
    c.check()
    x = c.out.double().cpu().numpy()
    for s in range(6):
        order = np.argsort(-x[s], kind="stable")[:20]
        order = np.sort(order[np.isfinite(x[s][order])])
        w = np.exp((x[s][order] - x[s].max()) / np.float64(np.float32(0.8)))
        assert int(kept[s]) == len(order)
        for j in range(2):
            v = float(u[2 * s + j]) * w.sum()
            if np.abs(w.cumsum() - v).min() > 1e-9 * w.sum():
                assert int(tokens[2 * s + j]) == order[(w.cumsum() <= v).sum()]
