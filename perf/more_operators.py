"""Cases of the operators that keep a long search within its cache and its answers within their rules, with plain forms of them:

  weights  ss_key_weights          the attention weight that every cached key receives in a step, added up over the steps
  evict    ss_kv_evict             keys of least accumulated weight leave a node; what stays is brought together in its first pages
  axes     ss_qk_norm_rope_axes,   norms and rotation where a token has a position on each of several axes (time, height, width),
           ss_kv_append_axes       in tensors, or on the way into the paged pool
  rules    ss_logit_rules          penalties of repeated tokens, biases and grammar masks on logits

A case is a dict of plain values; `prepare` makes its inputs on the GPU from a seed, `run` is one pass: in plain torch operations, or,
with `own`, through the library.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
D = 128                       # head dimension
PAGE = 16                     # tokens of a page
EPS = 1e-6
HEADS = [(12, 2), (28, 4), (32, 8), (16, 16), (8, 1)]


def listed():
    return [
        # one decoding step of a tiny tree: 8 candidates below one prompt; latency is all
        dict(name="weights_decode_8x12", op="weights", problems=1, paths=8, prefix=256, suffix=200, t_min=1, t_max=1, hq=12, hkv=2,
             last=0, decay=1.0, order=True),
        # a decoding step of a large search: 16 problems of 64 candidates, older weights fade
        dict(name="weights_decode_16x64", op="weights", problems=16, paths=64, prefix=512, suffix=480, t_min=1, t_max=1, hq=28, hkv=4,
             last=0, decay=0.97, order=False),
        # verification: steps of 64 tokens of 8 x 8 candidates over prompts of 4096 tokens
        dict(name="weights_verify_8x8x64", op="weights", problems=8, paths=8, prefix=4096, suffix=1024, t_min=64, t_max=64, hq=32, hkv=8,
             last=0, decay=1.0, order=True),
        # one long document, read in chunks of 128 tokens: the last 32 tokens say which of its keys matter
        dict(name="weights_window_131072", op="weights", problems=1, paths=1, prefix=0, suffix=131072, t_min=128, t_max=128, hq=32, hkv=8,
             last=32, decay=0.0, order=True),
        # a few short answers are cut to half
        dict(name="evict_16x1000", op="evict", nodes=16, length=1000, keep=0.5, sinks=4, recent=64, hkv=2, order=False),
        # a batch of sequences back into its budget, all of them cut before
        dict(name="evict_256x4096", op="evict", nodes=256, length=4096, keep=0.5, sinks=4, recent=128, hkv=4, order=True),
        # one long document, a quarter of it stays
        dict(name="evict_long_131072", op="evict", nodes=1, length=131072, keep=0.25, sinks=16, recent=1024, hkv=8, order=False),
        # a prompt with pictures, norms on, sections of the pairs for time, height and width
        dict(name="axes_rope_16384x32", op="axes", append=False, tokens=16384, hq=32, hkv=8, rot=128, interleaved=False, norm=True,
             cycled=False, axes=3, far=32768),
        # a decoding step of 512 candidates behind such prompts, keys into the pool; axes take turns over the pairs
        dict(name="axes_append_512x28", op="axes", append=True, tokens=512, hq=28, hkv=4, rot=128, interleaved=False, norm=False,
             cycled=True, axes=3, far=100000),
        # the next tokens of 8 sequences, repetition and frequency penalties; half-precision logits as an output layer leaves them
        dict(name="rules_8_bf16", op="rules", rows=8, vocab=151936, half=True, prompts=1, prompt=1000, history=600, repetition=1.1,
             frequency=0.2, presence=0.1, bias=0, masks=0),
        # the branching step of a large search: 922 sequences, some of them in a grammar, and a list of biases
        dict(name="rules_922", op="rules", rows=922, vocab=151936, half=False, prompts=16, prompt=512, history=480, repetition=1.05,
             frequency=0.0, presence=0.3, bias=300, masks=8),
        # sequences behind long documents
        dict(name="rules_64_long", op="rules", rows=64, vocab=151936, half=True, prompts=64, prompt=32000, history=4000, repetition=1.2,
             frequency=0.05, presence=0.0, bias=0, masks=2),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["weights", "evict", "axes", "rules"])
    hq, hkv = rng.choice(HEADS)
    if op == "weights":
        paths = rng.choice([1, 1, 2, 8, 40])
        t_max, problems = _log(rng, 1, 64), _log(rng, 1, max(1, 48 // paths))
        most = min(40000, 1000000 // (problems * hkv)) if paths == 1 and t_max < 8 else 2000
        return dict(op=op, problems=problems, paths=paths, prefix=16 * rng.randrange(0, 150) if paths > 1 else 0,
                    suffix=_log(rng, 1, most), t_min=rng.randint(1, t_max), t_max=t_max, hq=hq, hkv=hkv,
                    last=rng.choice([0, 0, 16]), decay=rng.choice([1.0, 0.97, 0.0]), order=rng.random() < 0.5)
    if op == "evict":
        nodes = _log(rng, 1, 200)
        return dict(op=op, nodes=nodes, length=_log(rng, 1, 150000 // nodes), keep=rng.choice([0.1, 0.25, 0.5, 0.9, 0.99]),
                    sinks=rng.choice([0, 4, 16]), recent=rng.choice([0, 32, 100]), hkv=hkv, order=rng.random() < 0.5)
    if op == "axes":
        return dict(op=op, append=rng.random() < 0.5, tokens=_log(rng, 1, 15000), hq=hq, hkv=hkv, rot=rng.choice([64, 96, 128, 128]),
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.6, cycled=rng.random() < 0.5, axes=rng.choice([2, 3, 3, 4]),
                    far=_log(rng, 100, 1000000))
    return dict(op=op, rows=_log(rng, 1, 400), vocab=rng.choice([151936, 32000, _log(rng, 50, 200000)]), half=rng.random() < 0.5,
                prompts=rng.choice([0, 1, 4]), prompt=_log(rng, 1, 8000), history=_log(rng, 1, 3000), repetition=rng.choice([1.0, 1.1, 1.3]),
                frequency=rng.choice([0.0, 0.2, -0.1]), presence=rng.choice([0.0, 0.5]), bias=rng.choice([0, 1, 40, 500]),
                masks=rng.choice([0, 1, 5]))


# ---- inputs ----------------------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


I32 = dict(dtype=torch.int32, device=DEV)
I64 = dict(dtype=torch.int64, device=DEV)


def _offsets(counts):
    at = [0]
    for x in counts:
        at.append(at[-1] + x)
    return at


def _sizes(case):
    """Lengths of a tree of one prompt a problem (the same for every seed): own tokens and step of every path."""
    r = random.Random("%(problems)d %(paths)d %(suffix)d %(t_min)d %(t_max)d" % case)
    n = case["problems"] * case["paths"]
    t = [r.randint(case["t_min"], case["t_max"]) for _ in range(n)]
    own_tokens = [case["suffix"] if n == 1 else r.randint(max(1, case["suffix"] // 2), case["suffix"]) for _ in range(n)]
    return own_tokens, t


def _tree(case, own_tokens, t, g):
    """One node per problem with its shared prefix, one leaf per path with its own tokens and the step's."""
    problems, paths, prefix = case["problems"], case["paths"], case["prefix"]
    n = problems * paths
    length = [prefix] * problems + [a + b for a, b in zip(own_tokens, t)]
    offsets, rows = _offsets([-(-x // PAGE) for x in length]), _offsets(t)
    s = dict(node_parent=torch.tensor([-1] * problems + [p // paths for p in range(n)], **I32), node_kv_len=torch.tensor(length, **I32),
             node_page_offsets=torch.tensor(offsets, **I64), node_pages=torch.randperm(offsets[-1], generator=g, **I32),
             path_leaf_node=torch.arange(problems, problems + n, **I32), path_q_len=torch.tensor(t, **I32),
             q_offsets=torch.tensor(rows, **I64), total_q=rows[-1], total_pages=offsets[-1], longest=max(length[problems:]), most=max(t))
    s["pool"] = torch.randn(offsets[-1], 2, case["hkv"], PAGE, D, generator=g, device=DEV, dtype=torch.bfloat16)
    return s


def _desc(B, s, case, q=None, lse=None):
    return B.make_attn_desc(num_q_heads=case["hq"], num_kv_heads=case["hkv"], kv_pool=s["pool"], node_parent=s["node_parent"],
                            node_kv_len=s["node_kv_len"], node_page_offsets=s["node_page_offsets"], node_pages=s["node_pages"],
                            total_node_pages=s["total_pages"], path_leaf_node=s["path_leaf_node"], path_q_len=s["path_q_len"],
                            q_offsets=s["q_offsets"], total_q=s["total_q"], q=q, out=None, lse=lse, max_depth=2)


def _lengths(case):
    """Lengths of the nodes of an eviction, and what is kept of each (the same for every seed)."""
    r = random.Random("%(nodes)d %(length)d" % case)
    n, most = case["nodes"], case["length"]
    length = [most if n == 1 else r.randint(max(1, most // 2), most) for _ in range(n)]
    return length, [max(1, int(x * case["keep"])) for x in length]


def _grid_positions(case, n, g):
    """[axes][n]: runs of a picture's tokens (32 a line, 32 lines a frame), each from a place of its own."""
    i = torch.arange(n, device=DEV)
    start = torch.randint(0, case["far"], (n // 1000 + 1,), generator=g, device=DEV)[i // 1000]
    steps = [i // 1024 % 64, i // 32 % 32, i % 32, i % 7]
    return torch.stack([start + steps[a] for a in range(case["axes"])]).to(torch.int32)


def _pair_axis(case):
    """Which axis turns which pair: turn by turn, or a section each, the first axis' half as long as the others'."""
    n, a = case["rot"] // 2, case["axes"]
    i = torch.arange(n, device=DEV)
    return (i % a if case["cycled"] else ((i * (2 * a - 1) // n + 1) // 2).clamp(max=a - 1)).to(torch.int32)


def _rules_sizes(case):
    """Lengths of prompts and histories, the prompt and mask of every row (the same for every seed)."""
    r = random.Random("%(rows)d %(prompt)d %(history)d" % case)
    n = case["rows"]
    prompt = [r.randint(max(1, case["prompt"] // 2), case["prompt"]) for _ in range(case["prompts"])]
    history = [r.choice([case["history"], r.randint(0, case["history"])]) for _ in range(n)]
    prompt_of = [i * case["prompts"] // n for i in range(n)] if case["prompts"] else []
    mask_of = [r.randrange(-1, case["masks"]) for _ in range(n)] if case["masks"] else []
    return prompt, history, prompt_of, mask_of


def _text(n, vocab, g):
    """Tokens as they come in text: few of them often."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab)) - 1).long().clamp(max=vocab - 1)
    return ((rank * 7919 + 13) % vocab).to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=case)
    op = case["op"]
    if op == "weights":
        own_tokens, t = _sizes(case)
        s.update(_tree(case, own_tokens, t, g))
        n, pages, hkv = s["total_q"], s["total_pages"], case["hkv"]
        s["q"] = 1.5 * torch.randn(n, case["hq"], D, generator=g, device=DEV, dtype=torch.bfloat16)
        s["lse"] = _log_sums(s)
        s["weights_in"] = torch.rand(pages, hkv, PAGE, generator=g, device=DEV) ** 4 if case["decay"] else None
        s["weights"] = torch.zeros(pages, hkv, PAGE, device=DEV)
        # numbers of the step's first tokens: keys have left the cache before
        s["path_order"] = torch.randint(50000, 100000, (len(t),), generator=g, **I32) if case["order"] else None
        s["order"] = torch.zeros(pages, hkv, PAGE, **I32) if case["order"] else None
        if own:
            from paper_2609_39334_b200 import binding as B
            s["desc"] = _desc(B, s, case, s["q"], s["lse"])
            s["step"] = B.make_key_weights(weights_out=s["weights"], weights_in=s["weights_in"], decay=case["decay"], last_tokens=case["last"],
                                           order=s["order"], path_order=s["path_order"])
            s["workspace"] = B.alloc_workspace(B.ss_key_weights_workspace_bytes(s["desc"], s["step"]), DEV)
    elif op == "evict":
        length, keep = _lengths(case)
        n, hkv = len(length), case["hkv"]
        tree = dict(case, problems=n, paths=1, prefix=0, hq=hkv)
        s.update(_tree(tree, [x - 1 for x in length], [1] * n, g))
        pages = s["total_pages"]
        s["nodes"] = torch.arange(n, 2 * n, **I32)                 # (the leaves)
        s["keep"] = torch.tensor(keep, **I32)
        w = torch.exp(2 * torch.randn(pages, hkv, PAGE, generator=g, device=DEV)) / 1000
        s["weights_in"] = torch.where(torch.rand(pages, hkv, PAGE, generator=g, device=DEV) < 0.05, 0, w)
        s["weights"], s["order"], s["order_in"] = torch.zeros_like(w), None, None
        if case["order"]:                                          # an eviction lies behind them: the older half in any order
            _, there, page, slot, head = _slots(s)
            i = torch.arange(s["longest"], device=DEV)
            old = (s["node_kv_len"].long()[s["nodes"].long()] // 2)[:, None, None]
            u = torch.rand(n, hkv, s["longest"], generator=g, device=DEV)
            order = torch.argsort(torch.where(i < old, u, 2.0 + i), dim=2)
            s["order_in"] = torch.zeros(pages, hkv, PAGE, **I32)
            at = there.expand_as(order)
            s["order_in"][page.expand_as(order)[at], head.expand_as(order)[at], slot.expand_as(order)[at]] = order[at].to(torch.int32)
            s["order"] = torch.zeros_like(s["order_in"])
        s["kv_len"] = s["node_kv_len"].clone()
        if own:
            from paper_2609_39334_b200 import binding as B
            s["desc"] = _desc(B, s, tree)
            s["cut"] = B.make_evict(nodes=s["nodes"], keep=s["keep"], weights=s["weights_in"], weights_out=s["weights"], order=s["order_in"],
                                    order_out=s["order"], kv_len_out=s["kv_len"], sinks=case["sinks"], recent=case["recent"],
                                    max_keys=s["longest"])
            s["workspace"] = B.alloc_workspace(B.ss_kv_evict_workspace_bytes(s["desc"], s["cut"]), DEV)
    elif op == "axes":
        n, hq, hkv = case["tokens"], case["hq"], case["hkv"]
        x = torch.randn(n, hq + 2 * hkv, D, generator=g, device=DEV, dtype=torch.bfloat16)
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        s["positions"], s["pair_axis"] = _grid_positions(case, n, g), _pair_axis(case)
        i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
        s["inv_freq"] = (1e6 ** (-2 * i / case["rot"])).float()
        w = (1 + 0.2 * torch.randn(2, D, generator=g, device=DEV)).bfloat16()
        s["wq"], s["wk"] = (w[0], w[1]) if case["norm"] else (None, None)
        s["q_out"] = torch.empty(n, hq, D, device=DEV, dtype=torch.bfloat16)
        if case["append"]:
            t = [1] * n if n <= 1024 else [n // 16 + (p < n % 16) for p in range(16)]
            r = random.Random(n)
            s.update(_tree(dict(case, problems=len(t), paths=1, prefix=0), [r.randint(0, 40) for _ in t], t, g))
        else:
            s["k_out"] = torch.empty(n, hkv, D, device=DEV, dtype=torch.bfloat16)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["rows"] = B.make_rows(q=s["q"], k=s["k"], v=s["v"] if case["append"] else None, q_out=s["q_out"], k_out=s.get("k_out"),
                                    inv_freq=s["inv_freq"], rot_dim=case["rot"], interleaved=case["interleaved"], q_weight=s["wq"],
                                    k_weight=s["wk"], eps=EPS)
            s["axes"] = B.make_axes(positions=s["positions"], pair_axis=s["pair_axis"])
            s["desc"] = _desc(B, s, case) if case["append"] else None
    else:
        n, v = case["rows"], case["vocab"]
        prompt, history, prompt_of, mask_of = _rules_sizes(case)
        x = 3 * torch.randn(n, v, generator=g, device=DEV)
        s["logits"] = x.bfloat16() if case["half"] else x
        s["out"] = torch.empty_like(s["logits"])
        s["history"], s["history_offsets"] = _text(sum(history), v, g), torch.tensor(_offsets(history), **I64)
        s["prompts"] = s["prompt_offsets"] = s["prompt_of"] = None
        if prompt:
            s["prompts"], s["prompt_offsets"] = _text(sum(prompt), v, g), torch.tensor(_offsets(prompt), **I64)
            s["prompt_of"] = torch.tensor(prompt_of, **I32)
        f32 = dict(dtype=torch.float32, device=DEV)
        s["repetition"], s["frequency"], s["presence"] = (torch.full((n,), case[x], **f32) for x in ("repetition", "frequency", "presence"))
        s["bias_tokens"] = s["bias_values"] = s["bias_offsets"] = s["bias_of"] = None
        if case["bias"]:                                           # two lists, taken in turn
            m = min(case["bias"], v)
            s["bias_tokens"] = torch.cat([torch.randperm(v, generator=g, **I32)[:m] for _ in range(2)])
            s["bias_values"] = 4 * torch.randn(2 * m, generator=g, device=DEV)
            s["bias_offsets"] = torch.tensor([0, m, 2 * m], **I64)
            s["bias_of"] = torch.arange(n, **I32) % 2
        s["masks"] = s["mask_of"] = None
        if case["masks"]:                                          # some grammars allow nearly all, some a handful
            share = torch.tensor([[0.95], [0.5], [0.1], [0.001]], device=DEV).repeat(-(-case["masks"] // 4), 1)[:case["masks"]]
            words = -(-v // 32)
            bits = torch.rand(case["masks"], words * 32, generator=g, device=DEV) < share
            power = 2 ** torch.arange(32, device=DEV)
            s["masks"] = (bits.view(-1, words, 32) * power).sum(2).to(torch.int32)
            s["mask_of"] = torch.tensor(mask_of, **I32)
        if own:
            from paper_2609_39334_b200 import binding as B
            s["rules"] = B.make_logit_rules(logits=s["logits"], out=s["out"], history=s["history"], history_offsets=s["history_offsets"],
                                            prompts=s["prompts"], prompt_offsets=s["prompt_offsets"], prompt_of=s["prompt_of"],
                                            repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                                            bias_tokens=s["bias_tokens"], bias_values=s["bias_values"], bias_offsets=s["bias_offsets"],
                                            bias_of=s["bias_of"], masks=s["masks"], mask_of=s["mask_of"])
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------------
def _padded_queries(s):
    """[path, kv head, head of the group, token of the step, dim], zeros behind a path's last token."""
    case = s["case"]
    n, most, hq, hkv = s["path_q_len"].numel(), s["most"], case["hq"], case["hkv"]
    path = torch.repeat_interleave(torch.arange(n, device=DEV), s["path_q_len"].long())
    t = torch.arange(s["total_q"], device=DEV) - s["q_offsets"][path]
    q = torch.zeros(n, most, hq, D, device=DEV)
    q[path, t] = s["q"].float()
    return q.view(n, most, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4), path, t


def _scores(s):
    """Scaled scores of every path's padded queries: with the prefix of its problem, [problem, kv head, path, group, token, key], and with
    its own keys, [path, kv head, group, token, key], -inf where a token does not see the key."""
    case = s["case"]
    problems, paths, prefix, hkv, longest = case["problems"], case["paths"], case["prefix"], case["hkv"], s["longest"]
    q, path, t = _padded_queries(s)
    n, _, group, most, _ = q.shape
    pages = s["node_pages"].long()
    first = s["node_page_offsets"]
    i = torch.arange(prefix, device=DEV)
    k = s["pool"][pages[first[:problems, None] + i // PAGE], 0, :, i % PAGE].float()          # [problem, key, kv head, dim]
    qp = q.reshape(problems, paths, hkv, group * most, D).transpose(1, 2).reshape(problems, hkv, paths * group * most, D)
    far = torch.matmul(qp, k.permute(0, 2, 3, 1)).view(problems, hkv, paths, group, most, prefix) / math.sqrt(D)
    j = torch.arange(longest, device=DEV)
    page = pages[(first[problems:problems + n, None] + j // PAGE).clamp(max=pages.numel() - 1)]
    k = s["pool"][page, 0, :, j % PAGE].float()
    near = torch.matmul(q.reshape(n, hkv, group * most, D), k.permute(0, 2, 3, 1)).view(n, hkv, group, most, longest) / math.sqrt(D)
    length, steps = s["node_kv_len"].long()[problems:, None, None], s["path_q_len"].long()[:, None, None]
    sees = j[None, None, :] <= length - steps + torch.arange(most, device=DEV)[None, :, None]
    near.masked_fill_(~sees[:, None, None], -math.inf)
    return far, near, path, t


def _log_sums(s):
    """What the attention leaves: [row, head], the logarithm of the row's sum of exponentials."""
    case = s["case"]
    far, near, path, t = _scores(s)
    n, hkv, group, most, _ = near.shape
    lse = torch.logsumexp(near, -1)
    if case["prefix"]:
        lse = torch.logaddexp(lse, torch.logsumexp(far, -1).transpose(1, 2).reshape(n, hkv, group, most))
    return lse.permute(0, 3, 1, 2).reshape(n, most, case["hq"])[path, t].contiguous()


def _plain_weights(s):
    case = s["case"]
    problems, paths, prefix, hkv = case["problems"], case["paths"], case["prefix"], case["hkv"]
    far, near, path, t = _scores(s)
    n, _, group, most, longest = near.shape
    # the row's log-sum, infinite where a row adds nothing: behind the step's end, or in front of its last tokens
    steps = s["path_q_len"].long()
    counts = t >= steps[path] - case["last"] if case["last"] else torch.ones_like(t, dtype=torch.bool)
    lse = torch.full((n, most, case["hq"]), math.inf, device=DEV)
    lse[path, t] = torch.where(counts[:, None], s["lse"], math.inf)
    lse = lse.view(n, most, hkv, group).permute(0, 2, 3, 1)                                   # [path, kv head, group, token]
    w_far = torch.exp(far - lse.reshape(problems, paths, hkv, group, most).transpose(1, 2)[..., None]).sum((2, 3, 4))
    w_near = torch.exp(near - lse[..., None]).sum((2, 3))                                     # [path, kv head, key]
    # where the sums go
    pages, first = s["node_pages"].long(), s["node_page_offsets"]
    h = torch.arange(hkv, device=DEV)[None, :, None]
    i = torch.arange(prefix, device=DEV)
    page = pages[first[:problems, None] + i // PAGE][:, None]
    before = s["weights_in"] if s["weights_in"] is not None else torch.zeros_like(s["weights"])
    s["weights"][page, h, i % PAGE] = before[page, h, i % PAGE] * case["decay"] + w_far
    j = torch.arange(longest, device=DEV)
    length = s["node_kv_len"].long()[problems:]
    page = pages[(first[problems:problems + n, None] + j // PAGE).clamp(max=pages.numel() - 1)][:, None].expand(n, hkv, longest)
    h, slot = h.expand(n, hkv, longest), (j % PAGE).expand(n, hkv, longest)
    at = j - (length - steps)[:, None]                                                        # number of a key in its step
    old = before[page, h, slot] * case["decay"]
    w_near += torch.where((at < 0)[:, None], old, 0)
    there = (j < length[:, None])[:, None].expand(n, hkv, longest)
    s["weights"][page[there], h[there], slot[there]] = w_near[there]
    if s["order"] is not None:
        new = there & (at >= 0)[:, None]
        s["order"][page[new], h[new], slot[new]] = (s["path_order"][:, None] + at).to(torch.int32)[:, None].expand(n, hkv, longest)[new]
    return s["weights"], s["order"]


def _slots(s):
    """Slots of the nodes of an eviction, padded to the longest: their lengths, which exist, page, place in it, head; [node, head, slot]."""
    i = torch.arange(s["longest"], device=DEV)[None, None, :]
    node = s["nodes"].long()
    length = s["node_kv_len"].long()[node][:, None, None]
    entry = (s["node_page_offsets"][node][:, None, None] + i // PAGE).clamp(max=s["total_pages"] - 1)
    return length, i < length, s["node_pages"].long()[entry], (i % PAGE).expand_as(entry), torch.arange(s["pool"].shape[2], device=DEV)[None, :, None]


def _plain_evict(s):
    case = s["case"]
    length, there, page, slot, head = _slots(s)
    shape = (length.shape[0], head.shape[1], there.shape[2])
    page, slot, head, there = page.expand(shape), slot.expand(shape), head.expand(shape), there.expand(shape)
    i = torch.arange(shape[2], device=DEV).expand(shape)
    order = torch.where(there, s["order_in"][page, head, slot].long() if s["order_in"] is not None else i, -1)
    stays = (order < case["sinks"]) | (order > order.amax(2, keepdim=True) - case["recent"])
    w = torch.where(stays, math.inf, s["weights_in"][page, head, slot])
    w = torch.where(there, w, -math.inf)
    keep = torch.minimum(s["keep"].long()[:, None, None], length)
    ranked = torch.sort(w, dim=2, descending=True, stable=True).indices
    kept = torch.zeros(shape, dtype=torch.bool, device=DEV).scatter_(2, ranked, i < keep)
    hole, moved = ~kept & (i < keep), kept & (i >= keep)           # as many of one as of the other in every row, both in order
    to, of = (page[hole], head[hole], slot[hole]), (page[moved], head[moved], slot[moved])
    s["pool"][to[0], :, to[1], to[2]] = s["pool"][of[0], :, of[1], of[2]]
    same = kept & ~moved
    at = (page[same], head[same], slot[same])
    s["weights"][at] = s["weights_in"][at]
    s["weights"][to] = s["weights_in"][of]
    if s["order"] is not None:
        s["order"][at] = s["order_in"][at]
        s["order"][to] = s["order_in"][of]
    s["kv_len"][s["nodes"].long()] = keep[:, 0, 0].to(torch.int32)
    return s["pool"], s["weights"], s["order"], s["kv_len"]


def _rotated(x, weight, s):
    """Head rows x [n, heads, 128], normalised where there is a weight, rotated to their positions; in 32 bits, angles in 64."""
    case = s["case"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = s["positions"].double()[s["pair_axis"].long()].T * s["inv_freq"].double()[None, :]
    c, n = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = case["rot"]
    turn, rest = y[..., :r], y[..., r:]
    if case["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turned = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = turn[..., :r // 2], turn[..., r // 2:]
        turned = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([turned, rest], -1).bfloat16()


def _plain_axes(s):
    s["q_out"].copy_(_rotated(s["q"], s["wq"], s))
    if not s["case"]["append"]:
        s["k_out"].copy_(_rotated(s["k"], s["wk"], s))
        return s["q_out"], s["k_out"]
    path = torch.repeat_interleave(torch.arange(s["path_q_len"].numel(), device=DEV), s["path_q_len"].long())
    leaf = s["path_leaf_node"].long()[path]
    at = s["node_kv_len"].long()[leaf] - s["path_q_len"].long()[path] + torch.arange(s["total_q"], device=DEV) - s["q_offsets"][path]
    page = s["node_pages"].long()[s["node_page_offsets"][leaf] + at // PAGE]
    s["pool"][page, 0, :, at % PAGE] = _rotated(s["k"], s["wk"], s)
    s["pool"][page, 1, :, at % PAGE] = s["v"]
    return s["q_out"], s["pool"]


def _plain_rules(s):
    x = s["logits"].float()
    n, v = x.shape
    length = s["history_offsets"][1:] - s["history_offsets"][:-1]
    row = torch.repeat_interleave(torch.arange(n, device=DEV), length)
    count = torch.zeros(n, v, device=DEV).index_put_((row, s["history"].long()), torch.ones((), device=DEV), accumulate=True)
    seen = count > 0
    if s["prompts"] is not None:
        m = s["prompt_offsets"].numel() - 1
        which = torch.repeat_interleave(torch.arange(m, device=DEV), s["prompt_offsets"][1:] - s["prompt_offsets"][:-1])
        in_prompt = torch.zeros(m, v, dtype=torch.bool, device=DEV).index_put_((which, s["prompts"].long()), torch.ones((), dtype=torch.bool, device=DEV))
        seen = seen | in_prompt[s["prompt_of"].long()]
    r = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count - torch.where(count > 0, s["presence"][:, None], 0)
    if s["bias_tokens"] is not None:
        m = s["bias_offsets"].numel() - 1
        which = torch.repeat_interleave(torch.arange(m, device=DEV), s["bias_offsets"][1:] - s["bias_offsets"][:-1])
        bias = torch.zeros(m, v, device=DEV).index_put_((which, s["bias_tokens"].long()), s["bias_values"])
        x = x + bias[s["bias_of"].long()]
    if s["masks"] is not None:
        token = torch.arange(v, device=DEV)
        allowed = (s["masks"][:, token // 32] >> (token % 32).to(torch.int32)) & 1 > 0
        of = s["mask_of"].long()
        x = torch.where((of < 0)[:, None] | allowed[of.clamp(min=0)], x, -math.inf)
    s["out"].copy_(x)
    return s["out"]


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2609_39334_b200 import binding as B
        if op == "weights":
            B.ss_key_weights(s["desc"], s["step"], s["workspace"])
            return s["weights"], s["order"]
        if op == "evict":
            B.ss_kv_evict(s["desc"], s["cut"], s["workspace"])
            return s["pool"], s["weights"], s["order"], s["kv_len"]
        if op == "axes":
            if s["case"]["append"]:
                B.ss_kv_append_axes(s["desc"], s["rows"], s["axes"])
                return s["q_out"], s["pool"]
            B.ss_qk_norm_rope_axes(s["rows"], s["axes"])
            return s["q_out"], s["k_out"]
        B.ss_logit_rules(s["rules"])
        return s["out"]
    if op == "weights":
        return _plain_weights(s)
    if op == "evict":
        return _plain_evict(s)
    if op == "axes":
        return _plain_axes(s)
    return _plain_rules(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "weights":
        own_tokens, t = _sizes(case)
        hq, hkv, prefix = case["hq"], case["hkv"], case["prefix"]
        used = [min(x, case["last"]) if case["last"] else x for x in t]
        keys = case["problems"] * prefix + sum(a + b for a, b in zip(own_tokens, t))
        pairs = sum(u * (prefix + a + b) for u, a, b in zip(used, own_tokens, t))
        arrays = (2 if case["decay"] else 1) * 4
        return dict(bytes=keys * hkv * (D * 2 + arrays) + sum(used) * hq * (D * 2 + 4) + keys // PAGE * 4 + (sum(t) * hkv * 4 if case["order"] else 0),
                    flops=pairs * hq * D * 2)
    if op == "evict":
        length, keep = _lengths(case)
        # of the keys that stay, those behind the first `keep` slots move; every weight is read, what stays is written
        moved = sum(k * (n - k) / n for n, k in zip(length, keep))
        arrays = 8 if case["order"] else 4
        return dict(bytes=int(case["hkv"] * (moved * D * 2 * 2 * 2 + (sum(length) + sum(keep)) * arrays)) + sum(length) // PAGE * 4,
                    flops=sum(length) * case["hkv"] * 4)
    if op == "axes":
        heads = case["hq"] + case["hkv"] * (2 if case["append"] else 1)
        n = case["tokens"]
        return dict(bytes=n * heads * D * 2 * 2 + n * case["axes"] * 4 + case["rot"] * 4 + (n * 24 if case["append"] else 0),
                    flops=n * (case["hq"] + case["hkv"]) * D * 7)
    prompt, history, _, mask_of = _rules_sizes(case)
    n, v = case["rows"], case["vocab"]
    return dict(bytes=n * v * (2 if case["half"] else 4) * 2 + (sum(prompt) + sum(history)) * 4 + case["masks"] * v // 8 + case["bias"] * 16 + n * 24,
                flops=n * v * 4)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------------
def _exact_weights(s):
    case = s["case"]
    own_tokens, t = _sizes(case)
    problems, hkv, group = case["problems"], case["hkv"], case["hq"] // case["hkv"]
    pages, first = s["node_pages"].long(), s["node_page_offsets"].tolist()
    out = torch.zeros(s["weights"].shape, dtype=torch.float64, device=DEV)
    order = s["order"].clone() if s["order"] is not None else None

    def keys(node):
        return s["pool"][pages[first[node]:first[node + 1]], 0].permute(1, 0, 2, 3).reshape(hkv, -1, D).double()

    def put(node, total, known):                                   # total [kv head, keys of the node's pages]
        mine = pages[first[node]:first[node + 1]]
        if mine.numel():
            old = s["weights_in"][mine].double() if s["weights_in"] is not None else torch.zeros(mine.numel(), hkv, PAGE, dtype=torch.float64, device=DEV)
            i = torch.arange(mine.numel() * PAGE, device=DEV).view(-1, 1, PAGE)
            new = total.view(hkv, -1, PAGE).transpose(0, 1) + torch.where(i < known, old * case["decay"], 0)
            out[mine] = torch.where(i < s["node_kv_len"][node], new, 0)

    scale, row = 1 / math.sqrt(D), 0
    for b in range(problems):
        shared = keys(b)
        total = torch.zeros(hkv, shared.shape[1], dtype=torch.float64, device=DEV)
        for p in range(b * case["paths"], (b + 1) * case["paths"]):
            u = min(t[p], case["last"]) if case["last"] else t[p]
            lo, hi = row + t[p] - u, row + t[p]
            q = s["q"][lo:hi].double().view(u, hkv, group, D).permute(1, 2, 0, 3).reshape(hkv, group * u, D)
            lse = s["lse"][lo:hi].double().view(u, hkv, group).permute(1, 2, 0).reshape(hkv, group * u, 1)
            total += torch.exp(q @ shared.transpose(1, 2) * scale - lse).sum(1)
            mine = keys(problems + p)
            step = torch.arange(t[p] - u, t[p], device=DEV).repeat(group)
            hidden = torch.arange(mine.shape[1], device=DEV)[None, :] > own_tokens[p] + step[:, None]
            put(problems + p, torch.exp((q @ mine.transpose(1, 2) * scale).masked_fill(hidden, -math.inf) - lse).sum(1), own_tokens[p])
            if order is not None:
                for x in range(t[p]):
                    at = own_tokens[p] + x
                    order[pages[first[problems + p] + at // PAGE], :, at % PAGE] = int(s["path_order"][p]) + x
            row = hi
        put(b, total, case["prefix"])
    return out, order


def _exact_evict(s):
    case = s["case"]
    length, keep = _lengths(case)
    n = len(length)
    hkv, pages, first = case["hkv"], s["node_pages"].cpu().numpy(), s["node_page_offsets"].tolist()
    w_in = s["weights_in"].cpu().numpy()
    o_in = s["order_in"].cpu().numpy() if s["order_in"] is not None else None
    w_out, o_out = np.zeros_like(w_in, dtype=np.float64), None if o_in is None else np.zeros_like(o_in)
    pool, kv_len = s["pool"].clone(), s["kv_len"].clone()
    to, of = [], []
    for e in range(n):
        mine = pages[first[n + e]:first[n + e + 1]]
        k = min(keep[e], length[e])
        kv_len[n + e] = k
        for h in range(hkv):
            w = w_in[mine, h].reshape(-1)[:length[e]]
            o = np.arange(length[e]) if o_in is None else o_in[mine, h].reshape(-1)[:length[e]].astype(np.int64)
            must = (o < case["sinks"]) | (o >= o.max() + 1 - case["recent"])
            best = np.argsort(-w, kind="stable")
            best = np.concatenate([np.flatnonzero(must), best[~must[best]]])[:k]      # those that must stay rank by slot among themselves
            stay = np.sort(best)
            free = np.setdiff1d(np.arange(k), stay)
            late = stay[stay >= k]
            src = np.arange(k)
            src[free] = late
            out = np.zeros(mine.size * PAGE)
            out[:k] = w[src]
            w_out[mine, h] = out.reshape(-1, PAGE)
            if o_out is not None:
                out = np.zeros(mine.size * PAGE, dtype=np.int64)
                out[:k] = o[src]
                o_out[mine, h] = out.reshape(-1, PAGE)
            to.append(np.stack([mine[free // PAGE], np.full(free.size, h), free % PAGE]))
            of.append(np.stack([mine[late // PAGE], np.full(late.size, h), late % PAGE]))
    to, of = (torch.tensor(np.concatenate(x, 1), device=DEV).long() for x in (to, of))
    pool[to[0], :, to[1], to[2]] = s["pool"][of[0], :, of[1], of[2]]
    return (pool.double(), torch.tensor(w_out, device=DEV), torch.tensor(o_out, device=DEV) if o_out is not None else None, kv_len)


def _exact_heads(x, weight, s):
    case = s["case"]
    z = x.double()
    if weight is not None:
        z = z / torch.sqrt(z.pow(2).sum(-1, keepdim=True) / D + EPS) * weight.double()
    half = case["rot"] // 2
    axis = s["pair_axis"].tolist()
    phi = torch.stack([s["positions"][axis[i]].double() * s["inv_freq"][i].double() for i in range(half)], 1)
    turn = torch.polar(torch.ones_like(phi), phi)[:, None, :]
    i = torch.arange(half, device=DEV)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    w = torch.complex(z[..., first], z[..., second]) * turn
    z[..., first], z[..., second] = w.real, w.imag
    return z


def _exact_rules(s):
    case = s["case"]
    prompt, history, prompt_of, mask_of = _rules_sizes(case)
    h, p = _offsets(history), _offsets(prompt)
    out = s["logits"].double()
    v = case["vocab"]
    allowed = None
    if case["masks"]:
        raw = s["masks"].cpu().numpy().astype("<i4").view(np.uint8).reshape(case["masks"], -1)
        allowed = torch.tensor(np.unpackbits(raw, axis=1, bitorder="little")[:, :v].astype(bool), device=DEV)
    for r in range(case["rows"]):
        x = out[r]
        count = torch.bincount(s["history"][h[r]:h[r + 1]].long(), minlength=v).double()
        seen = count > 0
        if prompt:
            seen = seen | (torch.bincount(s["prompts"][p[prompt_of[r]]:p[prompt_of[r] + 1]].long(), minlength=v) > 0)
        penalty = s["repetition"][r].double()
        x = torch.where(seen & (x > 0), x / penalty, torch.where(seen, x * penalty, x))
        x = x - s["frequency"][r].double() * count - s["presence"][r].double() * (count > 0)
        if case["bias"]:
            lo, hi = s["bias_offsets"][r % 2], s["bias_offsets"][r % 2 + 1]
            x[s["bias_tokens"][lo:hi].long()] += s["bias_values"][lo:hi].double()
        if mask_of and mask_of[r] >= 0:
            x[~allowed[mask_of[r]]] = -math.inf
        out[r] = x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "weights":
        return _exact_weights(s)
    if case["op"] == "evict":
        return _exact_evict(s)
    if case["op"] == "rules":
        return _exact_rules(s)
    q = _exact_heads(s["q"], s["wq"], s)
    if not case["append"]:
        return q, _exact_heads(s["k"], s["wk"], s)
    pool, k = s["pool"].double(), _exact_heads(s["k"], s["wk"], s)
    t, length = s["path_q_len"].tolist(), s["node_kv_len"].tolist()[len(s["path_q_len"]):]
    first, pages = s["node_page_offsets"].tolist(), s["node_pages"].tolist()
    place = [(pages[first[len(t) + p] + (length[p] - x + i) // PAGE], (length[p] - x + i) % PAGE) for p, x in enumerate(t) for i in range(x)]
    page, slot = torch.tensor(place, device=DEV).T
    pool[page, 0, :, slot], pool[page, 1, :, slot] = k, s["v"].double()
    return q, pool
