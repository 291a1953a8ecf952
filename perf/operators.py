"""Cases of the operators around the tree attention of a decoding or verification step, with plain forms of them:

  rope     ss_qk_norm_rope     norms of queries and keys per head with the position rotation
  append   ss_kv_append        keys and values of a step into the paged pool, rotated on the way (and the queries)
  draft    ss_draft_attention  attention of trees of drafted tokens over the paged cache
  sample   ss_filtered_sample  draws behind temperature, top-k, top-p and min-p from given random numbers

A case is a dict of plain values; `prepare` makes its inputs on the GPU from a seed, `run` is one pass: in plain torch operations, or,
with `own`, through the library.
"""
import math
import random

import torch

own = False

DEV = "cuda"
D = 128                       # head dimension
PAGE = 16                     # tokens of a page
EPS = 1e-6


def listed():
    return [
        # one decoding step of a tiny tree: 8 candidates, one token each (12 query and 2 key heads); latency is all
        dict(name="rope_decode_8x12", op="rope", tokens=8, hq=12, hkv=2, rot=128, interleaved=False, norm=True, far=4096),
        # verification of 256 steps of 16 to 128 tokens (28 and 4 heads), no norms, keys of a long context, pairs side by side
        dict(name="rope_verify_18437x28", op="rope", tokens=18437, hq=28, hkv=4, rot=64, interleaved=True, norm=False, far=1000000),
        # a prefill chunk of a model with query and key norms (32 and 8 heads)
        dict(name="rope_prefill_65536x32", op="rope", tokens=65536, hq=32, hkv=8, rot=128, interleaved=False, norm=True, far=65536),
        # expansion: 16 problems x 64 candidates, one token each, keys rotated into the pool, no norms
        dict(name="append_decode_16x64", op="append", problems=16, paths=64, prefix=512, suffix=480, t_min=1, t_max=1, hq=12, hkv=2,
             rot=128, interleaved=False, norm=False),
        # fine-grained verification: 8 x 32 candidates, steps of 16 to 128 tokens, norms on
        dict(name="append_verify_8x32", op="append", problems=8, paths=32, prefix=1024, suffix=448, t_min=16, t_max=128, hq=28, hkv=4,
             rot=128, interleaved=False, norm=True),
        # a large step: 8 x 128 candidates of 64 tokens each (32 and 8 heads)
        dict(name="append_verify_8x128", op="append", problems=8, paths=128, prefix=2048, suffix=256, t_min=64, t_max=64, hq=32, hkv=8,
             rot=128, interleaved=False, norm=True),
        # one sequence with a handful of drafted tokens: latency
        dict(name="draft_1x7", op="draft", problems=1, paths=1, prefix=0, suffix=300, t_min=7, t_max=7, hq=12, hkv=2),
        # a batch of sequences with trees of different sizes and cache lengths (28 and 4 heads)
        dict(name="draft_32x48", op="draft", problems=32, paths=1, prefix=0, suffix=4000, t_min=5, t_max=48, hq=28, hkv=4),
        # one very long context, 16 drafted tokens
        dict(name="draft_long_131072", op="draft", problems=1, paths=1, prefix=0, suffix=131072, t_min=16, t_max=16, hq=32, hkv=8),
        # candidates that share the prompt of their problem, each with a draft tree of 64 tokens
        dict(name="draft_8x8x64", op="draft", problems=8, paths=8, prefix=4096, suffix=1024, t_min=64, t_max=64, hq=32, hkv=8),
        # the next tokens of 8 sequences, a few draws each; half-precision logits as an output layer leaves them
        dict(name="sample_8_bf16", op="sample", rows=8, vocab=151936, half=True, most=4, top_k=50, top_p=0.95, min_p=0.0, temperature=0.8),
        # the branching step of a large search: 922 sequences, potentials up to 32, nucleus and minimum-probability filters
        dict(name="sample_922", op="sample", rows=922, vocab=151936, half=False, most=32, top_k=0, top_p=0.9, min_p=0.02, temperature=0.7),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "draft", "sample"])
    hq, hkv = rng.choice([(12, 2), (28, 4), (32, 8), (16, 16), (8, 1)])
    if op == "rope":
        return dict(op=op, tokens=_log(rng, 1, 50000), hq=hq, hkv=hkv, rot=rng.choice([32, 64, 96, 128, 128]),
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.6, far=_log(rng, 100, 1000000))
    if op == "append":
        t_max = _log(rng, 1, 128)
        return dict(op=op, problems=_log(rng, 1, 8), paths=_log(rng, 1, 64), prefix=16 * rng.randrange(0, 100),
                    suffix=_log(rng, 1, 700), t_min=rng.randint(1, t_max), t_max=t_max, hq=hq, hkv=hkv,
                    rot=rng.choice([64, 128, 128]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.6)
    if op == "draft":
        t_max = _log(rng, 1, 64)
        paths = rng.choice([1, 1, 2, 5])
        return dict(op=op, problems=_log(rng, 1, 12 // paths), paths=paths, prefix=16 * rng.randrange(0, 200) if paths > 1 else 0,
                    suffix=_log(rng, 1, 5000), t_min=rng.randint(1, t_max), t_max=t_max, hq=hq, hkv=hkv)
    return dict(op=op, rows=_log(rng, 1, 400), vocab=rng.choice([151936, 32000, _log(rng, 50, 200000)]), half=rng.random() < 0.5,
                most=_log(rng, 1, 64), top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.99, 0.95, 0.9, 0.5]),
                min_p=rng.choice([0.0, 0.0, 0.05, 0.2]), temperature=rng.choice([0.5, 0.7, 1.0, 1.3]))


# ---- inputs ----------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _frequencies(case, theta=1e6):
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    return (theta ** (-2 * i / case["rot"])).float()


def _weights(case, g):
    if not case["norm"]:
        return None, None
    w = 1 + 0.2 * torch.randn(2, D, generator=g, device=DEV)
    return w[0].bfloat16(), w[1].bfloat16()


def _packed(case, rows, g):
    """Queries, keys and values as views of one projection's output."""
    hq, hkv = case["hq"], case["hkv"]
    x = torch.randn(rows, hq + 2 * hkv, D, generator=g, device=DEV, dtype=torch.bfloat16)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _sizes(case):
    """Lengths of the tree of a case (the same for every seed): private tokens and step length of every path."""
    r = random.Random("%(problems)d %(paths)d %(suffix)d %(t_min)d %(t_max)d" % case)
    n = case["problems"] * case["paths"]
    t = [r.randint(case["t_min"], case["t_max"]) for _ in range(n)]
    own_tokens = [case["suffix"] if n == 1 else r.randint(max(1, case["suffix"] // 2), case["suffix"]) for _ in range(n)]
    return own_tokens, t


def _tree(case, g):
    """One node per problem with its shared prefix, one leaf per path with its own tokens and the step's."""
    own_tokens, t = _sizes(case)
    problems, paths, prefix = case["problems"], case["paths"], case["prefix"]
    n = problems * paths
    length = [prefix] * problems + [a + b for a, b in zip(own_tokens, t)]
    pages = [-(-x // PAGE) for x in length]
    offsets = [0]
    for x in pages:
        offsets.append(offsets[-1] + x)
    rows = [0]
    for x in t:
        rows.append(rows[-1] + x)
    i32 = dict(dtype=torch.int32, device=DEV)
    i64 = dict(dtype=torch.int64, device=DEV)
    s = dict(node_parent=torch.tensor([-1] * problems + [p // paths for p in range(n)], **i32), node_kv_len=torch.tensor(length, **i32),
             node_page_offsets=torch.tensor(offsets, **i64), node_pages=torch.randperm(offsets[-1], generator=g, **i32),
             path_leaf_node=torch.arange(problems, problems + n, **i32), path_q_len=torch.tensor(t, **i32),
             q_offsets=torch.tensor(rows, **i64), total_q=rows[-1], total_pages=offsets[-1], longest=prefix + max(length[problems:]),
             most=max(t))
    s["pool"] = torch.randn(offsets[-1], 2, case["hkv"], PAGE, D, generator=g, device=DEV, dtype=torch.bfloat16)
    return s


def _desc(B, s, case, q=None, out=None, lse=None):
    return B.make_attn_desc(num_q_heads=case["hq"], num_kv_heads=case["hkv"], kv_pool=s["pool"], node_parent=s["node_parent"],
                            node_kv_len=s["node_kv_len"], node_page_offsets=s["node_page_offsets"], node_pages=s["node_pages"],
                            total_node_pages=s["total_pages"], path_leaf_node=s["path_leaf_node"], path_q_len=s["path_q_len"],
                            q_offsets=s["q_offsets"], total_q=s["total_q"], q=q, out=out, lse=lse, max_depth=2)


def _draws(case):
    """Draws of every row: one, now and then none, some with a potential of up to case["most"]."""
    r = random.Random(case["rows"])
    return [r.choice([1] * 15 + [0]) if r.random() < 0.8 else r.randint(1, case["most"]) for _ in range(case["rows"] - 1)] + [1]


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=case)
    if case["op"] == "rope":
        n = case["tokens"]
        s["q"], s["k"], _ = _packed(case, n, g)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
        s["inv_freq"] = _frequencies(case)
        s["wq"], s["wk"] = _weights(case, g)
        s["q_out"] = torch.empty(n, case["hq"], D, device=DEV, dtype=torch.bfloat16)
        s["k_out"] = torch.empty(n, case["hkv"], D, device=DEV, dtype=torch.bfloat16)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["rows"] = B.make_rows(q=s["q"], k=s["k"], q_out=s["q_out"], k_out=s["k_out"], positions=s["positions"],
                                    inv_freq=s["inv_freq"], rot_dim=case["rot"], interleaved=case["interleaved"],
                                    q_weight=s["wq"], k_weight=s["wk"], eps=EPS)
    elif case["op"] == "append":
        s.update(_tree(case, g))
        s["q"], s["k"], s["v"] = _packed(case, s["total_q"], g)
        s["inv_freq"] = _frequencies(case)
        s["wq"], s["wk"] = _weights(case, g)
        s["q_out"] = torch.empty(s["total_q"], case["hq"], D, device=DEV, dtype=torch.bfloat16)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["desc"] = _desc(B, s, case)
            s["rows"] = B.make_rows(q=s["q"], k=s["k"], v=s["v"], q_out=s["q_out"], inv_freq=s["inv_freq"],
                                    rot_dim=case["rot"], interleaved=case["interleaved"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS)
    elif case["op"] == "draft":
        s.update(_tree(case, g))
        n = s["total_q"]
        s["q"] = torch.randn(n, case["hq"], D, generator=g, device=DEV, dtype=torch.bfloat16)
        t = torch.arange(n, device=DEV) - torch.repeat_interleave(s["q_offsets"][:-1], s["path_q_len"].long())
        # token t continues one of the tokens before it, or the cached text
        s["parent"] = ((torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * (t + 1)).floor().clamp(max=t) - 1).to(torch.int32)
        s["out"] = torch.empty(n, case["hq"], D, device=DEV, dtype=torch.bfloat16)
        s["lse"] = torch.empty(n, case["hq"], device=DEV, dtype=torch.float32)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["desc"] = _desc(B, s, case, s["q"], s["out"], s["lse"])
            s["workspace"] = B.alloc_workspace(B.ss_draft_attention_workspace_bytes(s["desc"]), DEV)
    else:
        n, v = case["rows"], case["vocab"]
        # an output layer's rows: noise, and a head that falls with the logarithm of its rank, steeper in some rows than in others
        logits = 1.5 * torch.randn(n, v, generator=g, device=DEV)
        m = min(v, 2000)
        stride = 7919 if v % 7919 else 7907                          # (prime: no token twice)
        at = (torch.randint(0, v, (n, 1), generator=g, device=DEV) + stride * torch.arange(m, device=DEV)) % v
        steep = 1 + 1.5 * torch.rand(n, 1, generator=g, device=DEV)
        logits.scatter_(1, at, 14 - steep * torch.log(torch.arange(1, m + 1, device=DEV, dtype=torch.float32)))
        s["logits"] = logits.bfloat16() if case["half"] else logits
        draws = _draws(case)
        s["most"], total = max(draws), sum(draws)
        s["draw_offsets"] = torch.tensor([sum(draws[:i]) for i in range(n + 1)], dtype=torch.int64, device=DEV)
        s["uniforms"] = torch.rand(total, generator=g, device=DEV)
        f32 = dict(dtype=torch.float32, device=DEV)
        s["temperature"] = torch.full((n,), case["temperature"], **f32)
        s["top_k"] = torch.full((n,), case["top_k"], dtype=torch.int32, device=DEV)
        s["top_p"] = torch.full((n,), case["top_p"], **f32)
        s["min_p"] = torch.full((n,), case["min_p"], **f32)
        s["tokens"] = torch.empty(total, dtype=torch.int32, device=DEV)
        s["seq"] = torch.empty(total, dtype=torch.int64, device=DEV)
        s["kept"] = torch.empty(n, dtype=torch.int32, device=DEV)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["desc"] = B.make_sample_desc(logits=s["logits"], draw_offsets=s["draw_offsets"], uniforms=s["uniforms"],
                                           temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                           tokens_out=s["tokens"], seq_out=s["seq"], kept_out=s["kept"])
            s["workspace"] = B.alloc_workspace(B.ss_filtered_sample_workspace_bytes(s["desc"]), DEV)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------------
def _rotated(x, weight, positions, inv_freq, case):
    """Head rows x [n, heads, 128], normalised where there is a weight, rotated to their positions; in 32 bits, angles in 64."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = positions.double()[:, None] * inv_freq.double()[None, :]
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = case["rot"]
    turn, rest = y[..., :r], y[..., r:]
    if case["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = turn[..., :r // 2], turn[..., r // 2:]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, rest], -1).bfloat16()


def _rows_of(s):
    """Path of every row, its number in the step, and the tokens in front of the path's leaf."""
    path = torch.repeat_interleave(torch.arange(s["path_q_len"].numel(), device=DEV), s["path_q_len"].long())
    t = torch.arange(s["total_q"], device=DEV) - s["q_offsets"][path]
    leaf = s["path_leaf_node"].long()
    before = s["node_kv_len"].long()[s["node_parent"].long()[leaf]]
    return path, t, leaf, before


def _plain_append(s):
    path, t, leaf, before = _rows_of(s)
    at = s["node_kv_len"].long()[leaf[path]] - s["path_q_len"].long()[path] + t
    positions = before[path] + at
    page = s["node_pages"].long()[s["node_page_offsets"][leaf[path]] + at // PAGE]
    k = _rotated(s["k"], s["wk"], positions, s["inv_freq"], s["case"])
    s["pool"][page, 0, :, at % PAGE] = k
    s["pool"][page, 1, :, at % PAGE] = s["v"]
    s["q_out"].copy_(_rotated(s["q"], s["wq"], positions, s["inv_freq"], s["case"]))
    return s["pool"], s["q_out"]


def _doubled(reach):
    return ((reach @ reach) > 0).float()


def _plain_draft(s):
    case = s["case"]
    hq, hkv = case["hq"], case["hkv"]
    path, t, leaf, before = _rows_of(s)
    n, most, longest = leaf.numel(), s["most"], s["longest"]
    # [path, draft, draft]: which drafted tokens a token continues, itself among them; paths of up to 128 links in seven doublings
    step = torch.zeros(n, most, most, device=DEV)
    child = s["parent"] >= 0
    step[path[child], t[child], s["parent"].long()[child]] = 1
    step += torch.eye(most, device=DEV)
    seen = _doubled(_doubled(_doubled(_doubled(_doubled(_doubled(_doubled(step)))))))
    # keys and values of every path, padded to the longest
    j = torch.arange(longest, device=DEV)[None, :]
    total = before + s["node_kv_len"].long()[leaf]
    node = torch.where(j < before[:, None], s["node_parent"].long()[leaf][:, None], leaf[:, None])
    inside = torch.where(j < before[:, None], j, j - before[:, None])
    there = j < total[:, None]
    page = s["node_pages"].long()[(s["node_page_offsets"][node] + inside // PAGE).clamp(max=s["total_pages"] - 1)]
    k = s["pool"][page, 0, :, inside % PAGE].float()               # [path, key, kv head, dim]
    v = torch.where(there[:, :, None, None], s["pool"][page, 1, :, inside % PAGE].float(), 0)
    draft = j - (total - s["path_q_len"].long())[:, None]
    q = torch.zeros(n, most, hq, D, device=DEV)
    q[path, t] = s["q"].float()
    q = q.view(n, most, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4)  # [path, kv head, head of the group, draft, dim]
    score = torch.einsum("phgtd,pkhd->phgtk", q, k) / math.sqrt(D)
    among = torch.gather(seen, 2, draft.clamp(0, most - 1)[:, None, :].expand(n, most, longest)) > 0
    visible = there[:, None, :] & ((draft < 0)[:, None, :] | among)
    score = torch.where(visible[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(score - top)
    total_e = e.sum(-1)
    out = torch.einsum("phgtk,pkhd->phgtd", e, v) / total_e[..., None]
    lse = torch.log(total_e) + top[..., 0]
    out = out.permute(0, 3, 1, 2, 4).reshape(n, most, hq, D)[path, t]
    lse = lse.permute(0, 3, 1, 2).reshape(n, most, hq)[path, t]
    return out.bfloat16(), lse


def _plain_sample(s):
    # in 64 bits: a draw next to the border between two tokens goes by the definition
    x, order = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    x = x.double()
    n, v = x.shape
    e = torch.exp((x - x[:, :1]) / s["temperature"].double()[:, None])
    rank = torch.arange(v, device=DEV)[None, :]
    limit = torch.where(s["top_k"] > 0, s["top_k"].long().clamp(max=v), v)
    kept = rank < limit[:, None]
    sums = torch.cumsum(torch.where(kept, e, 0), 1)
    p = s["top_p"].double()[:, None]
    kept &= (p >= 1) | (rank == 0) | (sums - e < p * sums[:, -1:])
    kept &= (rank == 0) | (e >= s["min_p"].double()[:, None])
    by_token = torch.zeros_like(e).scatter_(1, order, torch.where(kept, e, 0))
    sums = torch.cumsum(by_token, 1)
    count = s["draw_offsets"][1:] - s["draw_offsets"][:-1]
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), count)
    i = torch.arange(seq.numel(), device=DEV) - s["draw_offsets"][seq]
    u = torch.zeros(n, s["most"], dtype=torch.float64, device=DEV)
    u[seq, i] = s["uniforms"].double()
    token = torch.searchsorted(sums, u * sums[:, -1:], right=True)
    return token[seq, i].int(), seq, kept.sum(1).int()


def run(s):
    case = s["case"]
    if own:
        from paper_2609_39334_b200 import binding as B
        if case["op"] == "rope":
            B.ss_qk_norm_rope(s["rows"])
            return s["q_out"], s["k_out"]
        if case["op"] == "append":
            B.ss_kv_append(s["desc"], s["rows"])
            return s["pool"], s["q_out"]
        if case["op"] == "draft":
            B.ss_draft_attention(s["desc"], s["parent"], s["workspace"])
            return s["out"], s["lse"]
        B.ss_filtered_sample(s["desc"], s["workspace"])
        return s["tokens"], s["seq"], s["kept"]
    if case["op"] == "rope":
        s["q_out"].copy_(_rotated(s["q"], s["wq"], s["positions"], s["inv_freq"], case))
        s["k_out"].copy_(_rotated(s["k"], s["wk"], s["positions"], s["inv_freq"], case))
        return s["q_out"], s["k_out"]
    if case["op"] == "append":
        return _plain_append(s)
    if case["op"] == "draft":
        return _plain_draft(s)
    return _plain_sample(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "rope":
        rows = case["tokens"] * (case["hq"] + case["hkv"])
        return dict(bytes=rows * D * 2 * 2 + case["tokens"] * 4 + case["rot"] * 2 + (4 * D if case["norm"] else 0), flops=rows * D * 7)
    if case["op"] == "sample":
        return dict(bytes=case["rows"] * (case["vocab"] * (2 if case["half"] else 4) + 28) + sum(_draws(case)) * 16, flops=case["rows"] * case["vocab"] * 4)
    own_tokens, t = _sizes(case)
    n, hq, hkv = len(t), case["hq"], case["hkv"]
    if case["op"] == "append":
        rows = sum(t) * (hq + 2 * hkv)
        return dict(bytes=rows * D * 2 * 2 + n * 40, flops=sum(t) * (hq + hkv) * D * 7)
    keys = case["problems"] * case["prefix"] + sum(a + b for a, b in zip(own_tokens, t))
    pairs = sum(b * (case["prefix"] + a + b) for a, b in zip(own_tokens, t))
    return dict(bytes=keys * hkv * D * 2 * 2 + sum(t) * (hq * (D * 2 * 2 + 4) + 4) + keys // PAGE * 4, flops=pairs * hq * D * 4)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------------
def _exact_heads(x, weight, positions, inv_freq, case):
    z = x.double()
    if weight is not None:
        z = z / torch.sqrt(z.pow(2).sum(-1, keepdim=True) / D + EPS) * weight.double()
    half = case["rot"] // 2
    phi = torch.outer(positions.double(), inv_freq.double())
    turn = torch.polar(torch.ones_like(phi), phi)[:, None, :]
    i = torch.arange(half, device=DEV)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    w = torch.complex(z[..., first], z[..., second]) * turn
    z[..., first], z[..., second] = w.real, w.imag
    return z


def _exact_step_positions(s):
    own_tokens, t = _sizes(s["case"])
    return [s["case"]["prefix"] + a + i for a, b in zip(own_tokens, t) for i in range(b)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return tuple(_exact_heads(s[x], s["w" + x], s["positions"], s["inv_freq"], case) for x in "qk")
    if case["op"] == "append":
        own_tokens, t = _sizes(case)
        at = torch.tensor(_exact_step_positions(s), device=DEV)
        k, q = (_exact_heads(s[x], s["w" + x], at, s["inv_freq"], case) for x in "kq")
        pool = s["pool"].double()
        pages, first = s["node_pages"].tolist(), s["node_page_offsets"].tolist()
        place = [(pages[first[case["problems"] + p] + (a + i) // PAGE], (a + i) % PAGE)
                 for p, (a, b) in enumerate(zip(own_tokens, t)) for i in range(b)]
        page, slot = torch.tensor(place, device=DEV).T
        pool[page, 0, :, slot], pool[page, 1, :, slot] = k, s["v"].double()
        return pool, q
    if case["op"] == "draft":
        own_tokens, t = _sizes(case)
        group = case["hq"] // case["hkv"]
        outs, lses, row = [], [], 0
        parent = s["parent"].tolist()
        for p, (a, b) in enumerate(zip(own_tokens, t)):
            chain = [p // case["paths"], case["problems"] + p]
            length = [case["prefix"], a + b]
            kv = torch.cat([s["pool"][s["node_pages"][s["node_page_offsets"][x]:s["node_page_offsets"][x + 1]].long()]
                            .permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :y] for x, y in zip(chain, length)], 2).double()
            sees = torch.zeros(b, b, dtype=torch.bool)
            for i in range(b):
                if parent[row + i] >= 0:
                    sees[i] = sees[parent[row + i]]
                sees[i, i] = True
            cached = torch.ones(b, case["prefix"] + a, dtype=torch.bool)
            sees = torch.cat([cached, sees], 1).to(DEV)
            for h in range(case["hq"]):
                k, v = kv[0, h // group], kv[1, h // group]
                x = (s["q"][row:row + b, h].double() @ k.T * D ** -0.5).masked_fill(~sees, -math.inf)
                lse = torch.logsumexp(x, 1)
                outs.append(torch.exp(x - lse[:, None]) @ v)
                lses.append(lse)
            row += b
        outs = [torch.stack(outs[p * case["hq"]:(p + 1) * case["hq"]], 1) for p in range(len(t))]
        lses = [torch.stack(lses[p * case["hq"]:(p + 1) * case["hq"]], 1) for p in range(len(t))]
        return torch.cat(outs), torch.cat(lses)
    tokens, seqs, kepts = [], [], []
    first, u = s["draw_offsets"].tolist(), s["uniforms"].double()
    for r in range(case["rows"]):
        x = s["logits"][r].double()
        ids = torch.argsort(x, descending=True, stable=True)
        weight = torch.exp((x[ids] - x[ids[0]]) / s["temperature"][r].double())
        if case["top_k"]:
            ids, weight = ids[:case["top_k"]], weight[:case["top_k"]]
        n = ids.numel()
        if case["top_p"] < 1:
            n = min(n, int((torch.cumsum(weight, 0) < s["top_p"][r].double() * weight.sum()).sum()) + 1)
        n = max(1, min(n, int((weight >= s["min_p"][r].double()).sum())))
        ids, at = torch.sort(ids[:n])
        sums = torch.cumsum(weight[:n][at], 0)
        hit = (sums[None, :] <= u[first[r]:first[r + 1], None] * sums[-1]).sum(1)
        tokens.append(ids[hit].int())
        seqs.append(torch.full_like(hit, r))
        kepts.append(n)
    return torch.cat(tokens), torch.cat(seqs), torch.tensor(kepts, dtype=torch.int32, device=DEV)
