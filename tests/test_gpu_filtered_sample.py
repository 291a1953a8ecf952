"""ss_filtered_sample against a plain evaluation of its definition in 64 bits.

The call decides in fp64, the reference in 80 bits (2^-64: no error beside it).  A decision counts where the two sides of it are
further apart than near(V) of the sum.  A sum in fp64 of V terms by at least 512 threads, then by a tree: at most V / 512 + 32 roundings
of 2^-53 of it; a term: (|x| + 4) 2^-52 of itself for e^x (product with 1 / T, that quotient, the exponential), |x| 2^x at most 1
beside the largest term and log2 V on average (the entropy of the row): 60 2^-52 in all."""
import math

import numpy as np
import pytest
import torch

from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def near(V):
    return 2.0 ** -53 * (V / 512 + 32 + 120)


def reference(x, T, k, p, m):
    """(kept tokens by index, their weights, whether the filters' decision is clear) of one row of fp64 logits."""
    T, p, m = float(np.float32(T)), float(np.float32(p)), float(np.float32(m))
    NEAR = near(len(x))
    x = x.astype(np.longdouble)
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any() or not (T >= 0) or T == math.inf:
        return None, None, True
    order = np.argsort(-x, kind="stable")
    order = order[np.isfinite(x[order])]
    if T == 0:
        return order[:1], np.ones(1), True
    e = np.exp((x[order] - x[order[0]]) / T)
    n_k = min(k, len(order)) if k > 0 else len(order)
    n, clear = n_k, True
    if p < 1:
        sums = np.cumsum(e[:n_k])
        target = p * sums[-1]
        n_p = int((sums < target).sum()) + 1
        n = min(n, max(n_p, 1), n_k)
        # (whole numbers - weights of 1, and others too small to move a sum of them - add up without rounding in any order: exact)
        clear = bool(np.abs(sums - target).min() > NEAR * sums[-1]) or p <= 0 or bool((sums == np.rint(sums)).all())
    if m > 0:
        n_m = max(int((e >= m).sum()), 1)
        clear = clear and (n_m >= n or bool(np.abs(e - m).min() > NEAR) or m == 1)
        n = min(n, n_m)
    kept = np.sort(order[:n])
    return kept, np.exp((x[kept] - x[order[0]]) / T), clear


def check(logits, draws, T=1.0, k=0, p=1.0, m=0.0, seed=0, uniforms=None, stride=None, seq=True, kept=True, arrays=True, **kw):
    """Runs the call on `logits` (a CPU tensor) and compares every draw; returns the numbers of kept tokens."""
    n, V = logits.shape
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(draws)]).astype(np.int64)
    u = rng.random(off[-1]).astype(np.float32) if uniforms is None else np.asarray(uniforms, np.float32)
    per = [np.array(np.broadcast_to(np.asarray(a), (n,))) for a in (T, k, p, m)]
    full = torch.full((n, stride or V), float("nan"), dtype=logits.dtype, device=DEV)
    full[:, :V] = logits.to(DEV)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).to(DEV)
    tokens = torch.full((max(int(off[-1]), 1) + 2,), -7, dtype=torch.int32, device=DEV)
    seqs = torch.full((max(int(off[-1]), 1) + 2,), -7, dtype=torch.int64, device=DEV) if seq else None
    counts = torch.full((n,), -7, dtype=torch.int32, device=DEV) if kept else None
    params = dict(temperature=dev(per[0], torch.float32), top_k=dev(per[1], torch.int32), top_p=dev(per[2], torch.float32),
                  min_p=dev(per[3], torch.float32)) if arrays else dict(temperature=T, top_k=k, top_p=p, min_p=m)
    d = B.make_sample_desc(logits=full[:, :V], draw_offsets=dev(off, torch.int64), uniforms=dev(u if len(u) else np.zeros(1), torch.float32),
                           tokens_out=tokens, seq_out=seqs, kept_out=counts, **params)
    ws = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV)
    ws.fill_(0xEE)
    B.ss_filtered_sample(d, ws, **kw)
    torch.cuda.synchronize()
    got, x = tokens.cpu().numpy(), logits.double().numpy()
    assert (got[off[-1]:] == -7).all()
    if seq:
        assert np.array_equal(seqs.cpu().numpy()[:off[-1]], np.repeat(np.arange(n), draws))
    counted = counts.cpu().numpy() if kept else None
    unclear = 0
    for r in range(n):
        ids, w, clear = reference(x[r], *(a[r] for a in per))
        mine = got[off[r]:off[r + 1]]
        if ids is None:
            assert (mine == -1).all() and (counted is None or counted[r] == 0), r
            continue
        if not clear:
            unclear += 1
            continue
        if counted is not None:
            assert counted[r] == len(ids), (r, counted[r], len(ids))
        sums = np.cumsum(w)
        uu = u[off[r]:off[r + 1]].astype(np.float64)
        uu = np.where(uu < 1, np.maximum(uu, 0), 1.0)
        at = np.searchsorted(sums, uu * sums[-1], side="right")
        at = np.minimum(at, int((sums < sums[-1]).sum()))                  # (at the upper end: the last token that adds something)
        target = uu * sums[-1]
        close = np.minimum(np.abs(sums[at] - target), np.abs(sums[np.maximum(at - 1, 0)] - target)) <= near(V) * sums[-1]
        close &= (uu > 0) & (uu < 1)
        assert np.array_equal(mine[~close], ids[at][~close]), (r, mine[~close][:5], ids[at][~close][:5])
    assert unclear <= n // 8
    return counted


def rows(seed, n, V, kind="normal", dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g)
    if kind == "normal":
        x = 2 * x
    elif kind == "head":                                                    # as an output layer leaves them
        rank = torch.argsort(torch.argsort(torch.rand(n, V, generator=g), 1), 1).float() + 1
        x = x + 14 - (1 + 1.5 * torch.rand(n, 1, generator=g)) * torch.log(rank)
    elif kind == "grid":                                                    # many equal ones
        x = torch.round(2 * x)
    elif kind == "masked":
        x = 3 * x
        x[torch.rand(n, V, generator=g) < 0.6] = -math.inf
        x[:, V // 2] = 1.0
    elif kind == "sorted":
        x = torch.sort(3 * x, 1, descending=bool(seed & 1))[0]
    elif kind == "far":
        x = 3 * x + torch.tensor([3e4, -3e4, 0.0])[torch.arange(n) % 3][:, None]
    return x.to(dtype)


FILTERS = [dict(), dict(k=1), dict(k=50), dict(p=0.9), dict(p=0.99, T=1.3), dict(m=0.05), dict(k=40, p=0.95), dict(k=1000, p=0.5, m=0.02),
           dict(p=0.8, m=0.3), dict(T=0.0), dict(T=0.3, p=0.999)]


@pytest.mark.parametrize("V", [1, 2, 31, 257, 1000, 4099, 32000, 151936])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", range(len(FILTERS)))
def test_filters_and_sizes(V, dtype, f):
    n = 3 if V > 100000 else 7
    draws = [1, 40, 0, 3, 1, 1, 300][:n]
    for kind in ("normal", "head"):
        check(rows(V + f, n, V, kind, dtype), draws, seed=f, **FILTERS[f])


@pytest.mark.parametrize("kind", ["grid", "masked", "sorted", "far"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [600, 50001])
def test_kinds_of_rows(kind, dtype, V):
    for seed, f in enumerate(FILTERS):
        check(rows(seed, 6, V, kind, dtype), [1, 0, 17, 2, 1, 5], seed=seed, stride=V + 3, **f)


def test_parameters_by_row_and_as_numbers():
    x = rows(3, 64, 5000, "head")
    rng = np.random.default_rng(4)
    T, k = rng.choice([0.0, 0.2, 0.7, 1.0, 2.0], 64), rng.choice([0, 1, 5, 60, 4999, 5000, 10**6, -3], 64)
    p, m = rng.choice([0.0, 0.3, 0.9, 1.0, 1.5, np.nan], 64), rng.choice([0.0, 0.01, 0.5, 1.0, 1.5, np.nan, -1.0], 64)
    check(x, rng.integers(0, 4, 64), T, k, p, m)
    check(x, rng.integers(0, 4, 64), T, k, p, m, seq=False, kept=False)
    check(x, [2] * 64, 0.8, 30, 0.9, 0.05, arrays=False)


@pytest.mark.parametrize("V", [100, 40000])
def test_rows_without_a_distribution(V):
    x = rows(5, 8, V)
    x[0, V // 3] = math.nan
    x[1, 0] = math.inf
    x[2] = -math.inf
    x[3, V - 1] = -math.nan
    x[6, 5:] = -math.inf
    T = np.asarray([1, 1, 1, 1, -1.0, np.inf, 1.0, np.nan])
    for f in (dict(), dict(k=10), dict(p=0.9), dict(m=0.1)):
        kept = check(x, [2] * 8, T, **f)
        assert kept[6] > 0
    assert (check(x, [1] * 8, 0.0, p=0.5) == [0, 0, 0, 0, 1, 1, 1, 1]).all()


def test_all_equal_and_single_survivors():
    for V in (7, 5000, 151936):
        x = torch.zeros(3, V)
        x[1] = -5.25
        x[2, V // 2] = 200.0
        for f in (dict(p=0.9), dict(k=5), dict(k=5, p=0.5), dict(m=1.0), dict(p=0.999999), dict()):
            check(x, [50, 50, 50], **f)


def test_uniforms_at_the_ends():
    x = rows(6, 2, 3000)
    u = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, 0.5, 0.25]
    for f in FILTERS:
        check(x, [8, 0], uniforms=u, **f)


def test_tails_too_light_for_fixed_point():
    """A border among tokens of 1e-12 and less of the sum."""
    x = torch.cat([torch.zeros(2, 1), -20 - 12 * torch.rand(2, 30000, generator=torch.Generator().manual_seed(1))], 1)
    check(x, [3, 3], p=np.float32(1 - 2.0 ** -24))
    check(x, [3, 3], p=np.float32(1 - 2.0 ** -20))


def test_many_rows():
    x = rows(7, 700, 9000, "head")
    rng = np.random.default_rng(0)
    check(x, rng.integers(0, 6, 700), 0.9, 0, 0.92, 0.0)
    check(x.bfloat16(), rng.integers(0, 6, 700), 0.9, 100, 0.92, 0.001)


def test_unfiltered_draws_are_those_of_branch_sample():
    x = rows(8, 9, 20000, "head")
    n = 30
    off = torch.arange(0, 9 * n + 1, n, dtype=torch.int64, device=DEV)
    u = torch.rand(9 * n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    lg = x.to(DEV)
    a, b = [torch.empty(9 * n, dtype=torch.int32, device=DEV) for _ in range(2)]
    sa, sb = [torch.empty(9 * n, dtype=torch.int64, device=DEV) for _ in range(2)]
    B.ss_branch_sample(lg, off, u, 9, 20000, 0.8, a, sa)
    d = B.make_sample_desc(logits=lg, draw_offsets=off, uniforms=u, tokens_out=b, seq_out=sb, temperature=0.8)
    B.ss_filtered_sample(d, B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV))
    assert torch.equal(a, b) and torch.equal(sa, sb)


def test_graph_streams_and_offsets_that_do_not_start_at_zero():
    x = rows(9, 12, 30000, "head").to(DEV)
    off = torch.arange(5, 5 + 13 * 2, 2, dtype=torch.int64, device=DEV)
    u = torch.rand(40, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    tok = torch.full((40,), -7, dtype=torch.int32, device=DEV)
    d = B.make_sample_desc(logits=x, draw_offsets=off, uniforms=u, tokens_out=tok, top_k=40, top_p=0.9)
    ws = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV)
    B.ss_filtered_sample(d, ws)
    want = tok.clone()
    assert bool((want[:5] == -7).all()) and bool((want[5:29] >= 0).all()) and bool((want[29:] == -7).all())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.ss_filtered_sample(d, ws)
    for _ in range(3):
        tok.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, want)
    ws2 = torch.empty_like(ws)
    tok2 = torch.full_like(tok, -7)
    d2 = B.make_sample_desc(logits=x, draw_offsets=off, uniforms=u, tokens_out=tok2, top_k=40, top_p=0.9)
    torch.cuda.synchronize()
    for _ in range(5):
        B.ss_filtered_sample(d, ws)
        B.ss_filtered_sample(d2, ws2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(tok, want) and torch.equal(tok2, want)


@pytest.mark.parametrize("kind", ["normal", "grid", "head", "masked"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_keep_many(kind, dtype):
    """More kept tokens than fit a list: by top-k, by top-p, by min-p, by nothing, and with two of them."""
    V = 60001
    for seed, f in enumerate([dict(k=20000), dict(k=9000, T=1.5), dict(p=0.99, T=1.5), dict(p=0.7, T=4.0), dict(m=1e-4, T=2.0),
                              dict(k=20000, p=0.9, T=2.0), dict(p=0.99, m=0.003, T=1.5), dict(k=30000, m=0.01, T=1.5), dict(T=1.2), dict(k=59000, p=0.999, m=1e-5, T=3.0)]):
        check(rows(seed + 20, 3, V, kind, dtype), [3, 0, 40], seed=seed, **f)


def test_every_block_has_rows_and_parts():
    """Row numbers around whole rounds of one row a block: left-over rows are split, into many parts or none."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for n in (1, 2, sms, 2 * sms - 1, 2 * sms, 2 * sms + 1, 2 * sms + sms // 2, 2 * sms + sms + 3):
        check(rows(n, n, 9001, "head"), [1] * n, 0.9, 0, 0.9, 0.0, seed=n)
