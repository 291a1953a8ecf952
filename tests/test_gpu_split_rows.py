"""ss_filtered_sample on rows that several blocks share (few sequences, or those left over behind whole rounds), against the definition
in 64 bits: the parts of such a row see only what is theirs, and their sums are relative to what each of them saw."""
import math

import numpy as np
import pytest
import torch

import test_gpu_filtered_sample as plain
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V = 151936


def part_starts(n, dtype, vocab=V):
    """First tokens of the parts of a row where n rows are left over (a part's first 16 bytes are among those that it samples)."""
    per_vec = 4 if dtype == torch.float32 else 8
    blocks = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    parts = min(blocks // n, vocab // 4096, 32)
    assert parts >= 2 and vocab % per_vec == 0
    per = -(-(vocab // per_vec) // parts)
    return [p * per * per_vec for p in range(parts)]


def answers(row, n, T, p, m, u=(0.0, 0.5, 1 - 2.0 ** -24)):
    """(kept, tokens [n, len(u)]) of n copies of one row, top-p and min-p."""
    x = row.to(DEV).expand(n, V).contiguous()
    off = torch.arange(0, len(u) * n + 1, len(u), dtype=torch.int64, device=DEV)
    tokens, kept = torch.full((len(u) * n,), -7, dtype=torch.int32, device=DEV), torch.full((n,), -7, dtype=torch.int32, device=DEV)
    d = B.make_sample_desc(logits=x, draw_offsets=off, uniforms=torch.tensor(u, device=DEV).repeat(n), tokens_out=tokens, kept_out=kept,
                           temperature=T, top_p=p, min_p=m)
    B.ss_filtered_sample(d, B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV))
    return kept.cpu().numpy(), tokens.view(n, -1).cpu().numpy()


@pytest.mark.parametrize("n", [1, 9, 100, 148])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,top", [(0.014, 10.0), (0.014, 10.375), (0.01, 7.1875), (0.01, 7.375), (0.0121, 9.0), (0.014, 10.9375), (0.002, 5.0),
                                   (1e-5, 10.0)])
def test_parts_that_lie_a_float_s_exponent_apart(n, dtype, T, top):
    """Sums of parts whose largest terms are 2^1024 and more apart: the larger one is what counts, and top-p ends where it says also
    where min-p alone would keep more.  (Four equal tokens over noise 600 and more natural orders below them: whole numbers.)"""
    starts = part_starts(n, dtype)
    for at in {starts[len(starts) // 2 + len(starts) // 8], starts[-1]}:
        x = 0.001 * torch.randn(1, V, generator=torch.Generator().manual_seed(1))
        x[0, at:at + 4] = top
        for p, m, want in ((0.4, 0.1, 2), (0.4, 0.0, 2), (0.9, 0.1, 4), (0.2, 0.5, 1)):
            kept, tokens = answers(x.to(dtype), n, T, p, m)
            assert (kept == want).all(), (p, m, kept)
            assert (tokens == [at, at + want // 2, at + want - 1]).all()
        if n == 1:
            plain.check(x.to(dtype), [40], T, 0, 0.4, 0.1)
    if dtype == torch.float32:
        x[0, at + 1:at + 4] = top + T * math.log(0.05)
        kept, tokens = answers(x, n, T, 0.8, 0.02)                          # (weights 1, 0.05, 0.05, 0.05: the first is 0.87)
        assert (kept == 1).all() and (tokens == at).all()


def test_a_part_whose_largest_terms_its_sample_missed():
    """Two tokens that hold nearly all of the mass stand 65 powers of two above what their part's sample saw: their exponents are rounded
    to 2^-17, by 2^-18 downwards here (M log2(e) + 64 lies that far above a multiple of 2^-17), so the part's rough sum lacks 2.6e-6 of
    itself.  Top-p's target is a little above the first of them (1e-7 of it; 2^-24 of rounding in p)."""
    M, low = 0.700008749961853, -44.25
    starts = part_starts(1, torch.float32)
    x = -40 - torch.rand(1, V, generator=torch.Generator().manual_seed(3))
    a, b = starts[20], starts[21]
    x[0, a:b] = low - torch.rand(b - a, generator=torch.Generator().manual_seed(4))
    x[0, a:a + 4] = low                                                  # (sampled: what the part's sum is relative to)
    x[0, a + 1089] = x[0, a + 3753] = M                                  # (not sampled: vectors 272 and 938 of 1187, 32 of every 74 are)
    for beside in (1.0, 2.0, 3.0):
        x[0, 0] = M - beside
        total = float(np.exp(x[0].double().numpy() - float(np.float32(M))).sum())
        p = np.float32(1.0 / total)
        while float(p) * total <= 1 + 6e-8:
            p = np.nextafter(p, np.float32(1))
        assert float(p) * total < 1 + 3e-7
        assert (plain.check(x, [5], 1.0, 0, p, 0.0) == 2).all()


def times(n, vocab, dtype, **f):
    """Shortest of some calls on n rows, us."""
    x = plain.rows(n, n, vocab, "head").to(dtype).to(DEV)
    off, u = torch.arange(n + 1, device=DEV), torch.rand(n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(n))
    d = B.make_sample_desc(logits=x, draw_offsets=off, uniforms=u, tokens_out=torch.empty(n, dtype=torch.int32, device=DEV), **f)
    ws = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV)
    best = math.inf
    for _ in range(8):
        a, b = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        a.record()
        B.ss_filtered_sample(d, ws)
        b.record()
        torch.cuda.synchronize()
        best = min(best, 1e3 * a.elapsed_time(b))
    return best


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f", [dict(top_p=0.5), dict(top_k=2048, top_p=0.95)])
def test_rows_in_two_parts_fit_their_lists(dtype, f):
    """Half the SMs' worth of rows, in two parts each, go by their lists as one row more does, none of which is split: a list that
    overflows sends its row through passes over all of it, which takes ten times as long.  (Shortest of eight calls; 1.1 to 1 measured.)"""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert times(sms, V, dtype, **f) < 3 * times(sms + 1, V, dtype, **f)
    assert times(2 * sms // 3 + 1, V, dtype, **f) < 3 * times(sms + 1, V, dtype, **f)


@pytest.mark.parametrize("n", [1, 12, 99, 148])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_heads_and_low_temperatures(n, dtype):
    """Rows with a masked beginning, end or middle, and temperatures from where one token is kept to where hundreds are."""
    rng, vocab = np.random.default_rng(n), V if n < 99 else 33001
    x = plain.rows(n, n, vocab, "head").to(dtype)
    for r in range(n):
        cut = int(rng.integers(1, vocab - 1))
        if r % 3 == 0:
            x[r, :cut] = -math.inf
        elif r % 3 == 1:
            x[r, cut:] = -math.inf
        else:
            x[r, cut // 2:cut] = -math.inf
    T = rng.choice([1e-30, 1e-5, 0.003, 0.02, 0.1, 0.3, 1.0], n)
    draws = rng.integers(0, 3, n)
    plain.check(x, draws, T, 0, 0.9, 0.0)
    plain.check(x, draws, T, 0, 0.9, 0.05)
    plain.check(x, draws, T, rng.choice([0, 3, 50], n), 0.97, 0.01)


@pytest.mark.parametrize("n", [99, 100, 148])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_two_parts_a_row(n, dtype):
    x = plain.rows(n, n, 40001, "head").to(dtype)
    plain.check(x, [1] * n, 1.0, 0, 0.9, 0.0)
    plain.check(x, [1] * n, 0.8, 2048, 0.95, 0.0)
