"""What the bindings of the operators around the attention hand to the library, with tensors that only claim to be on a device: nothing is
launched and no pointer is followed."""
import ctypes

import pytest
import torch

from paper_2609_39334_b200 import binding as B
from paper_2609_39334_b200 import build as cuda_build


class Claimed:
    """A CPU tensor that says it is on a device."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return B.lib()


def sample(logits):
    n = logits.shape[0]
    return B.make_sample_desc(logits=Claimed(logits), draw_offsets=Claimed(torch.arange(n + 1)), uniforms=Claimed(torch.zeros(n)),
                              tokens_out=Claimed(torch.zeros(n, dtype=torch.int32)))


def workspace_rc(lib, d):
    out = ctypes.c_size_t(0)
    return lib.ss_filtered_sample_workspace_bytes(ctypes.byref(d), ctypes.byref(out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_logits_that_overlap_are_refused(lib, dtype):
    """One row expanded, or a window sliding over one buffer, is no matrix of rows `vocab` apart: it would be read as n rows behind each
    other, past the end of what there is."""
    row = torch.zeros(1, 1000, dtype=dtype)
    before = B.ss_launch_count()
    for logits in (row.expand(4, 1000), row.flatten().as_strided((4, 900), (1, 1)), row.flatten().as_strided((2, 501), (499, 1))):
        d = sample(logits)
        assert workspace_rc(lib, d) == B.SS_ERR_INVALID_ARG
        assert lib.ss_filtered_sample(ctypes.byref(d), 1 << 20, 1 << 40, None) == B.SS_ERR_INVALID_ARG
        with pytest.raises(B.SpecScaleError):
            B.ss_filtered_sample_workspace_bytes(d)
    assert B.ss_launch_count() == before


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_of_logits_that_are_taken(lib, dtype):
    """Whole rows, rows of a padded buffer, and a single row or none, whose stride says nothing."""
    full = torch.zeros(6, 1000, dtype=dtype)
    for logits, stride in ((full, 1000), (full[:, :900], 1000), (full[::2, 100:], 2000), (full[:1].expand(1, 1000), 1000),
                           (full.flatten().as_strided((1, 800), (0, 1)), 800), (full.flatten().as_strided((1, 800), (3, 1)), 800), (full[:0], 1000)):
        d = sample(logits)
        assert d.row_stride == stride and (d.n_seq, d.vocab) == tuple(logits.shape)
        assert workspace_rc(lib, d) == B.SS_OK
