"""ss_qk_norm_rope and ss_kv_append against a plain evaluation in 64 bits.

Tolerance: one rounding to bf16 is off by at most 2^-8 of the value.  Before it, in fp32: the products with weight and reciprocal
root (three roundings, a root good to 2^-22), the two products and the sum of a rotation (2^-23 of |y_a| + |y_b|), and a sine and
cosine whose argument was rounded once (off by at most pi 2^-24 + 2^-23): below 2^-20 of |y_a| + |y_b| in all."""
import itertools

import pytest
import torch

from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def turned(x, weight, pos, inv_freq, rot, interleaved, eps):
    """(exact rows, tolerance) of bf16 rows x [n, heads, 128] at positions pos."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    z, size = y.clone(), y.abs()
    if rot:
        f = pos.double()[:, None] * inv_freq.double()[None, :rot // 2]
        c, s = torch.cos(f)[:, None], torch.sin(f)[:, None]
        i = torch.arange(rot // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        both = y[..., a].abs() + y[..., b].abs()
        size[..., a], size[..., b] = both, both
    return z, 2.0 ** -8 * z.abs() + 2.0 ** -20 * size + 1e-38


def inv_freq(rot, theta=1e6):
    return (theta ** (-2 * torch.arange(rot // 2, dtype=torch.float64, device=DEV) / max(rot, 1))).float() if rot else None


def weights(on, g):
    return [(1 + 0.3 * torch.randn(128, generator=g, device=DEV)).bfloat16() if on else None for _ in range(2)]


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).bfloat16()


def close(got, want, tol):
    assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())


@pytest.mark.parametrize("n", [1, 2, 7, 300])
@pytest.mark.parametrize("heads", [(12, 2), (28, 4), (1, 1), (5, 3), (64, 8)])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (16, True), (96, False), (0, False)])
def test_norm_rope(n, heads, rot, interleaved):
    g = torch.Generator(device=DEV).manual_seed(n + 7 * rot + heads[0])
    hq, hk = heads
    x = randn(g, n, hq + hk + 1, 128)                                   # (a row stride that is not the heads')
    q, k = x[:, 1:1 + hq], x[:, 1 + hq:]
    pos = torch.randint(0, 1_000_000, (n,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = 0
    f = inv_freq(rot)
    for norm_q, norm_k in itertools.product((False, True), repeat=2):
        wq, wk = weights(norm_q, g)[0], weights(norm_k, g)[1]
        q_out, k_out = randn(g, n, hq, 128), randn(g, hk, n, 128).transpose(0, 1)     # (heads outermost)
        B.ss_qk_norm_rope(B.make_rows(q=q, k=k, q_out=q_out, k_out=k_out, positions=pos if rot else None, inv_freq=f, rot_dim=rot,
                                      interleaved=interleaved, q_weight=wq, k_weight=wk, eps=1e-6))
        for got, t, w in ((q_out, q, wq), (k_out, k, wk)):
            close(got, *turned(t, w, pos, f, rot, interleaved, 1e-6))
    # one of the two alone, in place
    want, tol = turned(q, None, pos, f, rot, interleaved, 1e-6)
    k_before = k.clone()
    B.ss_qk_norm_rope(B.make_rows(q=q, q_out=q, positions=pos if rot else None, inv_freq=f, rot_dim=rot, interleaved=interleaved))
    close(q, want, tol)
    assert torch.equal(k, k_before)


def test_norm_rope_many_rows_and_nothing():
    g = torch.Generator(device=DEV).manual_seed(5)
    n = 70001
    k = randn(g, n, 1, 128)
    pos = torch.randint(0, 1 << 30, (n,), generator=g, device=DEV, dtype=torch.int32)   # (no bits of the angle are lost)
    f = inv_freq(128)
    out = torch.empty_like(k)
    B.ss_qk_norm_rope(B.make_rows(k=k, k_out=out, positions=pos, inv_freq=f))
    close(out, *turned(k, None, pos, f, 128, False, 0.0))
    before = B.ss_launch_count()
    B.ss_qk_norm_rope(B.make_rows(k=k[:0], k_out=out[:0], positions=pos[:0], inv_freq=f))
    assert B.ss_launch_count() == before


def test_values_that_are_not_rotated_stay_as_they_are():
    """An infinity or NaN in a pair or behind the rotated part reaches no other value of an unnormalised row."""
    for interleaved in (False, True):
        g = torch.Generator(device=DEV).manual_seed(6)
        q = randn(g, 3, 4, 128)
        q[:, :, 70], q[:, :, 3], q[:, :, 127] = float("inf"), float("nan"), float("-inf")
        out = torch.empty_like(q)
        pos = torch.tensor([5, 6, 7], dtype=torch.int32, device=DEV)
        f = inv_freq(32)
        B.ss_qk_norm_rope(B.make_rows(q=q, q_out=out, positions=pos, inv_freq=f, interleaved=interleaved))
        assert torch.equal(out[..., 32:], q[..., 32:])
        touched = [2, 3] if interleaved else [3, 19]
        rest = [i for i in range(32) if i not in touched]
        assert bool(torch.isnan(out[..., touched]).all()) and bool(torch.isfinite(out[..., rest]).all())
        q[:, :, 3] = 1.0
        want, tol = turned(q, None, pos, f, 32, interleaved, 0.0)
        assert bool(((out.double() - want).abs() <= tol)[..., rest].all())


# ---- appending -------------------------------------------------------------------------------------------------------------------
def step(g, hq, hkv, lens, T, parents=None, indirect=False, pad_pool=False):
    """One root of 32 tokens, inner nodes `parents`, one leaf per path of lens[p] tokens (the step of T[p] tokens counted)."""
    n = len(lens)
    node_len = [32, 0, 16] + list(lens)
    node_par = [-1, 0, 1] + [(p % 4) - 1 for p in range(n)]             # below nothing, the root, the empty node or its child
    pages = [-(-x // 16) for x in node_len]
    off = [0] + list(itertools.accumulate(pages))
    rows = [0] + list(itertools.accumulate(T))
    i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
    n_pages = off[-1] + 3
    s = dict(node_par=node_par, node_len=node_len, off=off, rows=rows, T=list(T), n=n)
    s["pages"] = torch.randperm(n_pages, generator=g, device=DEV)[:off[-1]].to(torch.int32)
    s["src"] = [rows[-1] - r - t + 2 for r, t in zip(rows, T)] if indirect else rows[:-1]   # (backwards, two rows in front)
    n_rows = rows[-1] + (4 if indirect else 0)
    hp = hkv + (1 if pad_pool else 0)
    s["pool"] = randn(g, n_pages, 2, hp, 16, 128)
    s["q"], s["k"], s["v"] = randn(g, n_rows, hq, 128), randn(g, n_rows, hkv, 128), randn(g, n_rows, hkv, 128)
    pool = s["pool"]
    # (the descriptor only points to its tensors)
    s["keep"] = [torch.tensor(node_par, **i32), torch.tensor(node_len, **i32), torch.tensor(off, **i64), torch.arange(3, 3 + n, **i32),
                 torch.tensor(list(T), **i32), torch.tensor(rows, **i64), torch.tensor(s["src"], **i64)]
    node_parent, node_kv_len, offsets, leaf, steps, q_offsets, src = s["keep"]
    s["desc"] = B.make_attn_desc(
        num_q_heads=hq, num_kv_heads=hkv, k_pool=pool[:, 0], v_pool=pool[:, 1], num_pages=n_pages, kv_page_stride=pool.stride(0),
        kv_head_stride=2048, kv_token_stride=128, node_parent=node_parent, node_kv_len=node_kv_len,
        node_page_offsets=offsets, node_pages=s["pages"], total_node_pages=off[-1], path_leaf_node=leaf,
        path_q_len=steps, q_offsets=q_offsets, total_q=rows[-1], q=None, out=None, q_src_offsets=src if indirect else None,
        q_src_rows=n_rows if indirect else 0)
    return s


def chain_start(s, p):
    before, a = 0, s["node_par"][3 + p]
    while a >= 0:
        before += s["node_len"][a]
        a = s["node_par"][a]
    return before


@pytest.mark.parametrize("hq,hkv", [(12, 2), (8, 8), (4, 1)])
@pytest.mark.parametrize("kind", ["decode", "steps", "longer_than_leaf", "indirect", "many"])
@pytest.mark.parametrize("norm,rot,interleaved", [(True, 128, False), (False, 64, True), (False, 0, False)])
def test_append(hq, hkv, kind, norm, rot, interleaved):
    g = torch.Generator(device=DEV).manual_seed(hq + rot)
    r = torch.Generator().manual_seed(3)
    n = {"many": 150}.get(kind, 9)
    T = [1] * n if kind == "decode" else torch.randint(1, 70, (n,), generator=r).tolist()
    lens = [t + x for t, x in zip(T, torch.randint(0, 50, (n,), generator=r).tolist())]
    if kind == "longer_than_leaf":
        lens[2], lens[4] = T[2] - 1, 0
    s = step(g, hq, hkv, lens, T, indirect=kind == "indirect", pad_pool=kind == "steps")
    f = inv_freq(rot)
    wq, wk = weights(norm, g)
    q_out = randn(g, *s["q"].shape)
    want_pool, want_q, q_written = s["pool"].double(), torch.zeros(q_out.shape, dtype=torch.float64, device=DEV), []
    tol_pool = torch.zeros_like(want_pool)
    tol_q = torch.zeros_like(want_q)
    before_q = q_out.clone()
    for p in range(n):
        rows = torch.arange(s["src"][p], s["src"][p] + T[p], device=DEV)
        at = torch.arange(T[p], device=DEV) + lens[p] - T[p]
        pos = at + chain_start(s, p)
        k, k_tol = turned(s["k"][rows], wk, pos, f, rot, interleaved, 1e-6)
        want_q[rows], tol_q[rows] = turned(s["q"][rows], wq, pos, f, rot, interleaved, 1e-6)
        q_written += rows.tolist()
        ok = at >= 0
        page = s["pages"].long()[s["off"][3 + p] + at[ok] // 16]
        want_pool[page, 0, :hkv, at[ok] % 16], tol_pool[page, 0, :hkv, at[ok] % 16] = k[ok], k_tol[ok]
        want_pool[page, 1, :hkv, at[ok] % 16] = s["v"][rows][ok].double()
    B.ss_kv_append(s["desc"], B.make_rows(q=s["q"], k=s["k"], v=s["v"], q_out=q_out, inv_freq=f, rot_dim=rot, interleaved=interleaved,
                                          q_weight=wq, k_weight=wk))
    close(s["pool"], want_pool, tol_pool)                                # untouched slots: equal
    w = torch.zeros(q_out.shape[0], dtype=torch.bool)
    w[q_written] = True
    close(q_out[w.to(DEV)], want_q[w.to(DEV)], tol_q[w.to(DEV)])
    assert torch.equal(q_out[~w.to(DEV)], before_q[~w.to(DEV)])         # rows of no path: left alone


def test_append_given_positions_live_paths_and_bad_indices():
    g = torch.Generator(device=DEV).manual_seed(11)
    T, lens = [3, 4, 5, 2], [20, 33, 5, 18]
    s = step(g, 4, 2, lens, T)
    f = inv_freq(128)
    pos = torch.randint(0, 5000, (s["rows"][-1],), generator=g, device=DEV, dtype=torch.int32)
    pages = s["pages"]
    bad = s["off"][3 + 1] + 2                                             # the third page of path 1 (tokens 32 and on) is nowhere
    pages[bad] = 1 << 20
    live = torch.tensor([3], dtype=torch.int32, device=DEV)
    s["desc"].num_paths_dev = live.data_ptr()
    want = s["pool"].clone()
    for p in range(3):
        for t in range(T[p]):
            at, row = lens[p] - T[p] + t, s["rows"][p] + t
            if p == 1 and at >= 32:
                continue
            page = int(pages[s["off"][3 + p] + at // 16])
            k, _ = turned(s["k"][row:row + 1], None, pos[row:row + 1], f, 128, False, 0.0)
            want[page, 0, :, at % 16] = k[0].float().bfloat16()
            want[page, 1, :, at % 16] = s["v"][row]
    B.ss_kv_append(s["desc"], B.make_rows(k=s["k"], v=s["v"], inv_freq=f, positions=pos))
    assert bool(((s["pool"].float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs()).all())
    assert torch.equal(s["pool"][:, 1], want[:, 1])


def test_rows_in_a_graph_and_on_another_stream():
    g = torch.Generator(device=DEV).manual_seed(12)
    s = step(g, 4, 2, [20, 33], [3, 4])
    f = inv_freq(128)
    q_out = torch.empty_like(s["q"])
    rows = B.make_rows(q=s["q"], k=s["k"], v=s["v"], q_out=q_out, inv_freq=f)
    B.ss_kv_append(s["desc"], rows)
    first = s["pool"].clone(), q_out.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.ss_kv_append(s["desc"], rows)
    s["pool"].zero_()
    q_out.zero_()
    graph.replay()
    touched = first[0] != 0
    torch.cuda.synchronize()
    assert torch.equal(q_out, first[1])
    assert torch.equal(s["pool"][s["pool"] != 0], first[0][s["pool"] != 0]) and bool(touched.any())
    side.wait_stream(torch.cuda.current_stream())
    q_out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    B.ss_kv_append(s["desc"], rows, stream=side)
    side.synchronize()
    assert torch.equal(q_out, first[1])
