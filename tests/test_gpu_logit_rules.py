"""ss_logit_rules against a plain evaluation in 64 bits.

Tolerance: the quotient or product, the product with the count, its difference, the presence's and the bias: five roundings of fp32, 2^-24 each
of what is added up (|x|, |x r| or |x / r|, |frequency| c, |presence|, |bias|); then one rounding to bf16 (2^-8 of the result) where that is the type."""
import itertools

import numpy as np
import pytest
import torch

from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32, I64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)


def csr(lists, dtype=torch.int32):
    off = [0] + list(itertools.accumulate(len(x) for x in lists))
    return torch.tensor([y for x in lists for y in x], dtype=dtype, device=DEV), torch.tensor(off, **I64)


class Case:
    def __init__(self, seed, n, vocab, half, history=None, prompts=None, prompt_of=None, r=1.0, f=0.0, p=0.0, bias=None, bias_of=None, masks=None,
                 mask_of=None, in_place=False, stride=0, shift=0, out_shift=None, arrays=False):
        g = torch.Generator(device=DEV).manual_seed(seed)
        dtype = torch.bfloat16 if half else torch.float32
        self.n, self.vocab, self.half = n, vocab, half
        stride = max(stride, vocab)

        def rows(shift):
            return torch.full((n * stride + shift + 8,), 7.0, dtype=dtype, device=DEV)[shift:shift + n * stride].as_strided((n, vocab), (stride, 1))
        self.x = rows(shift)
        self.x.copy_(3 * torch.randn(n, vocab, generator=g, device=DEV))
        self.out = self.x if in_place else rows(shift if out_shift is None else out_shift)
        self.x0 = self.x.double()
        self.history, self.prompts, self.bias, self.masks = history, prompts, bias, masks
        self.prompt_of = prompt_of if prompt_of is not None else list(range(n))
        self.bias_of = bias_of if bias_of is not None else list(range(n))
        self.mask_of = mask_of if mask_of is not None else list(range(n))
        rep = lambda v: [float(v)] * n if not isinstance(v, (list, tuple)) else [float(y) for y in v]  # noqa: E731
        self.r, self.f, self.p = rep(r), rep(f), rep(p)
        kw = {}
        for name, v in (("repetition", r), ("frequency", f), ("presence", p)):
            kw[name] = torch.tensor(rep(v), device=DEV) if arrays or isinstance(v, (list, tuple)) else float(v)
        if history is not None:
            kw["history"], kw["history_offsets"] = csr(history)
        if prompts is not None:
            kw["prompts"], kw["prompt_offsets"] = csr(prompts)
            kw["prompt_of"] = torch.tensor(prompt_of, **I32) if prompt_of is not None else None
        if bias is not None:
            kw["bias_tokens"], kw["bias_offsets"] = csr([[t for t, _ in x] for x in bias])
            kw["bias_values"] = csr([[v for _, v in x] for x in bias], torch.float32)[0]
            kw["bias_of"] = torch.tensor(bias_of, **I32) if bias_of is not None else None
        if masks is not None:
            words = -(-vocab // 32)
            bits = np.zeros((len(masks), words * 32), dtype=bool)
            bits[:, :vocab] = masks
            bits[:, vocab:] = np.arange(bits.shape[1] - vocab) % 2 == 0      # (behind the vocabulary: anything)
            packed = np.packbits(bits, axis=1, bitorder="little").view("<i4").copy()
            kw["masks"] = torch.tensor(packed, device=DEV)
            kw["mask_of"] = torch.tensor(mask_of, **I32) if mask_of is not None else None
        self.rules = B.make_logit_rules(logits=self.x, out=None if in_place else self.out, **kw)

    def expected(self):
        x = self.x0.cpu().numpy().copy()
        size = np.zeros_like(x)
        v = self.vocab
        for s in range(self.n):
            hist = np.array([t for t in (self.history[s] if self.history else []) if 0 <= t < v], dtype=np.int64)
            count = np.bincount(hist, minlength=v).astype(float)
            seen = count > 0
            if self.prompts is not None and 0 <= self.prompt_of[s] < len(self.prompts):
                for t in self.prompts[self.prompt_of[s]]:
                    if 0 <= t < v:
                        seen[t] = True
            r, f, p = (np.float32(a[s]) for a in (self.r, self.f, self.p))
            r = np.float64(r) if r > 0 else 1.0
            f, p = np.float64(f), np.float64(p)
            with np.errstate(invalid="ignore", over="ignore"):
                y = np.where(seen, np.where(x[s] > 0, x[s] / r, x[s] * r), x[s])
                size[s] = np.where(seen & (r != 1), np.abs(y), 0)
                y = np.where(count > 0, y - f * count - p, y)
                size[s] = np.where(count > 0, size[s] + np.abs(y) + np.abs(f * count) + abs(p), size[s])
                if self.bias is not None and 0 <= self.bias_of[s] < len(self.bias):
                    for t, b in dict(self.bias[self.bias_of[s]]).items():
                        if 0 <= t < v:
                            y[t] += np.float64(np.float32(b))
                            size[s, t] += abs(y[t]) + abs(b)
                if self.masks is not None and 0 <= self.mask_of[s] < len(self.masks):
                    y[~self.masks[self.mask_of[s]]] = -np.inf
                    size[s][~self.masks[self.mask_of[s]]] = 0
            x[s] = y
        return torch.tensor(x, device=DEV), torch.tensor(size, device=DEV)

    def check(self):
        want, size = self.expected()
        got = self.out.double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        fin = torch.isfinite(want)
        assert torch.equal(got[~fin].nan_to_num(5), want[~fin].nan_to_num(5))
        tol = 5 * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() * (size > 0) if self.half else 0)
        bad = fin & ((got - want).abs() > tol)
        assert not bad.any(), (bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


def text(r, n, v):
    return [int(x) for x in np.minimum(v - 1, np.floor(np.exp(r.random(n) * np.log(v))) - 1)]


def everything(seed, n, v, half, **kw):
    r = np.random.default_rng(seed)
    masks = r.random((3, v)) < np.array([[0.9], [0.5], [0.02]])
    return Case(seed, n, v, half, history=[text(r, int(x), v) for x in r.integers(0, 300, n)], prompts=[text(r, 200, v), [], text(r, 3000, v)],
                prompt_of=[int(x) for x in r.integers(-1, 4, n)], r=[1.0, 1.3, 0.7][:n] + [1.1] * (n - 3), f=[0.2] * n, p=[0.5] * n,
                bias=[[(int(t), float(b)) for t, b in zip(r.integers(0, v, 50), r.normal(size=50))], [], [(v - 1, 2.5), (0, -100.0)]],
                bias_of=[int(x) for x in r.integers(-1, 4, n)], masks=masks, mask_of=[int(x) for x in r.integers(-1, 4, n)], **kw)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("v", [1, 5, 31, 33, 1000, 8191, 8192, 8193, 8205, 20011, 151936])
def test_everything_together(v, half):
    for in_place in (False, True):
        c = everything(v, 7, v, half, in_place=in_place)
        B.ss_logit_rules(c.rules)
        c.check()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("stride,shift,out_shift", [(0, 1, 1), (0, 3, 0), (16411, 5, 5), (16411, 0, 2), (16416, 4, 4)])
def test_rows_anywhere(stride, shift, out_shift, half):
    c = everything(stride + shift, 6, 16401, half, stride=stride, shift=shift, out_shift=out_shift)
    whole = c.out.as_strided((c.n * c.out.stride(0) + out_shift,), (1,), 0).clone() if stride else None
    B.ss_logit_rules(c.rules)
    c.check()
    if stride:                                                    # what lies between the rows is left alone
        now = c.out.as_strided(whole.shape, (1,), 0)
        gap = torch.ones(whole.shape, dtype=torch.bool, device=DEV)
        for s in range(c.n):
            gap[out_shift + s * stride:out_shift + s * stride + c.vocab] = False
        assert torch.equal(now[gap], whole[gap])


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("kw", [
    dict(), dict(r=1.2), dict(f=0.5), dict(p=0.5), dict(r=0.0), dict(r=-1.0), dict(r=float("nan")), dict(f=-0.5, p=-1.0), dict(r=1.2, arrays=True)])
def test_penalties_alone(kw, half):
    r = np.random.default_rng(3)
    for in_place in (False, True):
        c = Case(3, 4, 9000, half, history=[text(r, 100, 9000), [], [8999] * 5000, [0, 0, -1, 9000, 1 << 30, -(1 << 31)]],
                 prompts=[[7, 7, 8191], text(r, 50, 9000)], prompt_of=[0, 1, 5, -1], in_place=in_place, **kw)
        B.ss_logit_rules(c.rules)
        c.check()


@pytest.mark.parametrize("half", [False, True])
def test_prompt_list_and_mask_of_the_rows_number(half):
    r = np.random.default_rng(4)
    v = 1003
    c = Case(4, 3, v, half, prompts=[text(r, 50, v), text(r, 60, v)], r=1.5, bias=[[(5, 1.0)], [(6, float("-inf")), (7, float("inf"))]],
             masks=r.random((2, v)) < 0.5)
    B.ss_logit_rules(c.rules)
    c.check()


@pytest.mark.parametrize("half", [False, True])
def test_a_token_twice_in_a_bias_list_takes_the_last_entry(half):
    v = 700
    lists = [[(3, 1.0), (9, 2.0), (3, -4.0), (9, 2.5), (3, 0.5), (-1, 9.0), (700, 9.0)] + [(i % 50, float(i)) for i in range(2000)]]
    c = Case(5, 3, v, half, bias=lists, bias_of=[0, 0, -1])
    B.ss_logit_rules(c.rules)
    c.check()


@pytest.mark.parametrize("half", [False, True])
def test_odd_logits(half):
    v = 300
    c = Case(6, 2, v, half, history=[list(range(0, 300, 2)) * 2, list(range(300))], r=1.3, f=0.1, p=0.2)
    for s in range(2):
        for i, x in enumerate((float("nan"), float("inf"), float("-inf"), 0.0, -0.0, 1e-38, -3e38, 3e38)):
            c.x[s, 20 * s + i] = x
    c.x0 = c.x.double()
    B.ss_logit_rules(c.rules)
    want, _ = c.expected()
    over = want.abs() > 3.3e38                                    # (out of range: an infinity)
    got = c.out.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    rest = ~over & ~torch.isnan(want)
    assert torch.isinf(got[over]).all() and ((got - want)[rest].abs() <= (2.0 ** -8 if half else 2.0 ** -21) * (want[rest].abs() + 1)).all()


def test_a_row_with_nothing_allowed_draws_nothing():
    v = 2000
    c = Case(7, 3, v, False, masks=np.array([[False] * v, [i == 77 for i in range(v)]]), mask_of=[0, 1, -1])
    B.ss_logit_rules(c.rules)
    c.check()
    tokens, kept = torch.zeros(3, **I32), torch.zeros(3, **I32)
    d = B.make_sample_desc(logits=c.out, draw_offsets=torch.arange(4, **I64), uniforms=torch.full((3,), 0.5, device=DEV), tokens_out=tokens,
                           kept_out=kept)
    B.ss_filtered_sample(d, B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(d), DEV))
    assert tokens[:2].tolist() == [-1, 77] and kept.tolist() == [0, 1, v]


def test_nothing_to_do_and_long_histories():
    B.ss_logit_rules(B.make_logit_rules(logits=torch.zeros(0, 50, device=DEV), history=torch.zeros(0, **I32), history_offsets=torch.zeros(1, **I64)))
    r = np.random.default_rng(8)
    c = Case(8, 2, 40000, True, history=[text(r, 70000, 40000), text(r, 3, 40000)], prompts=[text(r, 100001, 40000)], prompt_of=[0, 0], r=1.1, f=0.01)
    B.ss_logit_rules(c.rules)
    c.check()


def test_graph_and_another_stream():
    c = everything(9, 5, 5000, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.ss_logit_rules(c.rules)
    s.synchronize()
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.ss_logit_rules(c.rules)
    for _ in range(2):
        c.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        c.check()
