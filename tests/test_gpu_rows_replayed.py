"""ss_qk_norm_rope and ss_kv_append captured into a graph: every place of the step is written again by every replay, and no other."""
import pytest
import torch

import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def places(s, lens):
    """(page, slot) of every token of the step, in the order of its rows."""
    page, slot = [], []
    for p, t in enumerate(s["T"]):
        at = torch.arange(lens[p] - t, lens[p], device=DEV)
        page.append(s["pages"].long()[s["off"][3 + p] + at // 16])
        slot.append(at % 16)
    return torch.cat(page), torch.cat(slot)


@pytest.mark.parametrize("T", [[3, 4], [1, 1, 1], [70, 5, 33]])
def test_every_replay_writes_every_place(T):
    g = torch.Generator(device=DEV).manual_seed(sum(T))
    lens = [t + 17 * i for i, t in enumerate(T)]
    s = rows_test.step(g, 4, 2, lens, T)
    f = rows_test.inv_freq(128)
    wq, wk = rows_test.weights(True, g)
    q_out = torch.empty_like(s["q"])
    rows = B.make_rows(q=s["q"], k=s["k"], v=s["v"], q_out=q_out, inv_freq=f, q_weight=wq, k_weight=wk)
    page, slot = places(s, lens)
    assert len(set(zip(page.tolist(), slot.tolist()))) == sum(T)
    pos = torch.cat([torch.arange(n - t, n, device=DEV) + rows_test.chain_start(s, p) for p, (n, t) in enumerate(zip(lens, T))])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.ss_kv_append(s["desc"], rows)
    for round_ in range(3):
        if round_:                                                       # other rows in the same buffers
            for name in ("q", "k", "v"):
                s[name].copy_(rows_test.randn(g, *s[name].shape))
        s["pool"].fill_(7.0)
        q_out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        rows_test.close(s["pool"][page, 0, :, slot], *rows_test.turned(s["k"], wk, pos, f, 128, False, 1e-6))
        assert torch.equal(s["pool"][page, 1, :, slot], s["v"])
        rows_test.close(q_out, *rows_test.turned(s["q"], wq, pos, f, 128, False, 1e-6))
        s["pool"][page, :, :, slot] = 7.0
        assert bool((s["pool"] == 7).all())


def test_rotation_replayed():
    g = torch.Generator(device=DEV).manual_seed(3)
    n = 300
    q, k = rows_test.randn(g, n, 12, 128), rows_test.randn(g, n, 2, 128)
    pos = torch.randint(0, 100000, (n,), generator=g, device=DEV, dtype=torch.int32)
    f = rows_test.inv_freq(64)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    rows = B.make_rows(q=q, k=k, q_out=q_out, k_out=k_out, positions=pos, inv_freq=f, interleaved=True)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.ss_qk_norm_rope(rows)
    for _ in range(2):
        pos.copy_(torch.randint(0, 100000, (n,), generator=g, device=DEV, dtype=torch.int32))
        q_out.fill_(7.0)
        k_out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        rows_test.close(q_out, *rows_test.turned(q, None, pos, f, 64, True, 0.0))
        rows_test.close(k_out, *rows_test.turned(k, None, pos, f, 64, True, 0.0))
