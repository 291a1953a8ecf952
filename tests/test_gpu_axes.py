"""ss_qk_norm_rope_axes and ss_kv_append_axes against a plain evaluation in 64 bits (tolerance: see test_gpu_rows), and against the forms
without axes, whose results they give bit for bit where every axis says the same."""
import pytest
import torch

import test_gpu_draft_attention as draft
import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


def turned(x, weight, positions, pair_axis, inv_freq, rot, interleaved, eps):
    """As test_gpu_rows.turned; the frequency of a pair at its axis' position is that of position 1 at the product."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    z, size = y.clone(), y.abs()
    if rot:
        axis = pair_axis.long().clamp(0, positions.shape[0] - 1)
        f = (positions.double()[axis] * inv_freq.double()[:rot // 2, None]).T[:, None]
        c, s = torch.cos(f), torch.sin(f)
        i = torch.arange(rot // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        both = y[..., a].abs() + y[..., b].abs()
        size[..., a], size[..., b] = both, both
    return z, 2.0 ** -8 * z.abs() + 2.0 ** -20 * size + 1e-38


@pytest.mark.parametrize("n", [1, 5, 300, 9001])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, True), (96, False), (16, False), (0, False)])
def test_norm_rope(n, axes, rot, interleaved):
    g = torch.Generator(device=DEV).manual_seed(n + axes + rot)
    hq, hk = 5, 2
    x = rows_test.randn(g, n, hq + hk, 128)
    q, k = x[:, :hq], x[:, hq:]
    f = rows_test.inv_freq(rot)
    positions = torch.randint(-50, 1_000_000, (axes, n + 3), generator=g, **I32)[:, :n]
    pair_axis = torch.randint(-1, axes + 1, (max(rot // 2, 1),), generator=g, **I32)      # (the ends count as the nearer axis)
    wq, wk = rows_test.weights(True, g)
    q_out, k_out = rows_test.randn(g, n, hq, 128), rows_test.randn(g, hk, n, 128).transpose(0, 1)
    r = B.make_rows(q=q, k=k, q_out=q_out, k_out=k_out, inv_freq=f, rot_dim=rot, interleaved=interleaved, q_weight=wq, eps=1e-6)
    B.ss_qk_norm_rope_axes(r, B.make_axes(positions=positions, pair_axis=pair_axis))
    rows_test.close(q_out, *turned(q, wq, positions, pair_axis, f, rot, interleaved, 1e-6))
    rows_test.close(k_out, *turned(k, None, positions, pair_axis, f, rot, interleaved, 1e-6))


@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, True)])
def test_equal_axes_are_one(rot, interleaved):
    g = torch.Generator(device=DEV).manual_seed(3)
    n, hq, hk = 1000, 4, 2
    x = rows_test.randn(g, n, hq + hk, 128)
    pos = torch.randint(0, 1_000_000, (n,), generator=g, **I32)
    f = rows_test.inv_freq(rot)
    outs = []
    for axes in (0, 3):
        q_out, k_out = rows_test.randn(g, n, hq, 128), rows_test.randn(g, n, hk, 128)
        r = B.make_rows(q=x[:, :hq], k=x[:, hq:], q_out=q_out, k_out=k_out, positions=None if axes else pos, inv_freq=f, interleaved=interleaved)
        if axes:                                                  # one row of positions for all axes
            B.ss_qk_norm_rope_axes(r, B.make_axes(positions=pos[None].expand(axes, n), pair_axis=torch.arange(rot // 2, **I32) % axes))
        else:
            B.ss_qk_norm_rope(r)
        outs.append((q_out, k_out))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("queries", [False, True])
@pytest.mark.parametrize("kw", [dict(chains=[[64, 20], [64, 30], [64, 9]], T=[4, 9, 1], shared=(0,)),
                                dict(chains=[[16, 3], [0]], T=[100, 1], src=[5, 200]),
                                dict(chains=[[0] for _ in range(400)], T=[1 + p % 3 for p in range(400)])])
def test_append(kw, queries):
    c = draft.Case(4, 6, 2, **kw)
    g = torch.Generator(device=DEV).manual_seed(5)
    n = c.q.shape[0]
    x = rows_test.randn(g, n, 6 + 4, 128)
    q, k, v = x[:, :6], x[:, 6:8], x[:, 8:]
    positions = torch.randint(0, 100000, (3, n), generator=g, **I32)
    pair_axis = torch.randint(0, 3, (64,), generator=g, **I32)
    f, (_, wk) = rows_test.inv_freq(128), rows_test.weights(True, g)
    q_out = torch.full((n, 6, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    r = B.make_rows(q=q if queries else None, k=k, v=v, q_out=q_out if queries else None, inv_freq=f, k_weight=wk)
    before = c.pool.clone()
    B.ss_kv_append_axes(c.desc, r, B.make_axes(positions=positions, pair_axis=pair_axis))
    written, rows_used = torch.zeros(c.pool.shape[0], 16, dtype=torch.bool, device=DEV), torch.zeros(n, dtype=torch.bool, device=DEV)
    for p, t in enumerate(c.T):
        rr = torch.arange(c.src[p], c.src[p] + t, device=DEV)
        leaf = c.chain[p][-1]
        at = torch.arange(c.lens[leaf] - t, c.lens[leaf], device=DEV)
        page = c.pages.long()[c.off[leaf] + at // 16]
        rows_test.close(c.pool[page, 0, :, at % 16], *turned(k[rr], wk, positions[:, rr], pair_axis, f, 128, False, 1e-6))
        assert torch.equal(c.pool[page, 1, :, at % 16], v[rr])
        written[page, at % 16] = True
        rows_used[rr] = True
        if queries:
            rows_test.close(q_out[rr], *turned(q[rr], None, positions[:, rr], pair_axis, f, 128, False, 1e-6))
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(c.pool.permute(0, 3, 1, 2, 4)[~written], before.permute(0, 3, 1, 2, 4)[~written])
    assert (q_out[~rows_used] == 7.0).all() if queries else (q_out == 7.0).all()


def test_graph():
    g = torch.Generator(device=DEV).manual_seed(6)
    n = 64
    q = rows_test.randn(g, n, 4, 128)
    positions, pair_axis, f = torch.randint(0, 1000, (3, n), generator=g, **I32), torch.arange(64, **I32) % 3, rows_test.inv_freq(128)
    q_out = torch.empty_like(q)
    r, a = B.make_rows(q=q, q_out=q_out, inv_freq=f), B.make_axes(positions=positions, pair_axis=pair_axis)
    B.ss_qk_norm_rope_axes(r, a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ss_qk_norm_rope_axes(r, a)
    positions.add_(17)
    graph.replay()
    torch.cuda.synchronize()
    rows_test.close(q_out, *turned(q, None, positions, pair_axis, f, 128, False, 1e-6))
