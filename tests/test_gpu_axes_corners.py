"""ss_kv_append_axes where the number of paths is known on the device alone."""
import pytest
import torch

import test_gpu_axes as axes
import test_gpu_draft_attention as draft
import test_gpu_rows as rows_test
from paper_2609_39334_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("live", [0, 1, 2, 3])
def test_live_paths_are_counted_on_the_device(live):
    c = draft.Case(51, 6, 2, chains=[[64, 20], [64, 30], [64, 9]], T=[4, 9, 1], shared=(0,))
    g = torch.Generator(device=DEV).manual_seed(52)
    n = c.q.shape[0]
    x = rows_test.randn(g, n, 6 + 4, 128)
    positions, pair_axis = torch.randint(0, 100000, (3, n), generator=g, **I32), torch.randint(0, 3, (64,), generator=g, **I32)
    f, q_out = rows_test.inv_freq(128), torch.full((n, 6, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    count = torch.tensor([live], **I32)
    c.desc.num_paths_dev = count.data_ptr()
    before = c.pool.clone()
    B.ss_kv_append_axes(c.desc, B.make_rows(q=x[:, :6], k=x[:, 6:8], v=x[:, 8:], q_out=q_out, inv_freq=f),
                        B.make_axes(positions=positions, pair_axis=pair_axis))
    written = torch.zeros(c.pool.shape[0], 16, dtype=torch.bool, device=DEV)
    for p in range(live):
        rr = torch.arange(c.rows[p], c.rows[p + 1], device=DEV)
        leaf = c.chain[p][-1]
        at = torch.arange(c.lens[leaf] - c.T[p], c.lens[leaf], device=DEV)
        page = c.pages.long()[c.off[leaf] + at // 16]
        rows_test.close(c.pool[page, 0, :, at % 16], *axes.turned(x[rr, 6:8], None, positions[:, rr], pair_axis, f, 128, False, 1e-6))
        assert torch.equal(c.pool[page, 1, :, at % 16], x[rr, 8:])
        rows_test.close(q_out[rr], *axes.turned(x[rr, :6], None, positions[:, rr], pair_axis, f, 128, False, 1e-6))
        written[page, at % 16] = True
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(c.pool.permute(0, 3, 1, 2, 4)[~written], before.permute(0, 3, 1, 2, 4)[~written])
    assert (q_out[c.rows[live]:] == 7.0).all()
