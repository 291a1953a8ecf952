"""Refusals of the operators around the attention on the host: nothing is launched and no pointer is followed."""
import ctypes

import pytest

from paper_2609_39334_b200 import binding as B
from paper_2609_39334_b200 import build as cuda_build

OK = 1 << 20                      # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return B.lib()


@pytest.fixture(autouse=True)
def nothing_launched(lib):
    before = B.ss_launch_count()
    yield
    assert B.ss_launch_count() == before


def rows(**kw):
    r = B.ss_rows_t()
    r.struct_size = ctypes.sizeof(B.ss_rows_t)
    r.num_q_heads, r.num_kv_heads, r.head_dim, r.rot_dim, r.n_rows, r.eps = 12, 2, 128, 128, 10, 1e-6
    r.inv_freq = r.positions = r.q = r.q_out = r.k = OK
    r.q_row_stride = r.q_out_row_stride = r.k_row_stride = r.v_row_stride = r.k_out_row_stride = 2048
    r.q_head_stride = r.q_out_head_stride = r.k_head_stride = r.v_head_stride = r.k_out_head_stride = 128
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def desc(**kw):
    d = B.ss_attn_desc_t()
    d.struct_size = ctypes.sizeof(B.ss_attn_desc_t)
    d.num_q_heads, d.num_kv_heads, d.head_dim, d.page_size = 12, 2, 128, 16
    d.kv_page_stride, d.kv_head_stride, d.kv_token_stride = 2 * 2 * 2048, 2048, 128
    d.num_nodes, d.num_paths, d.total_q, d.total_node_pages, d.num_pages = 10, 8, 8, 100, 100
    for n in ("k_pool", "v_pool", "node_parent", "node_kv_len", "node_page_offsets", "node_pages", "path_leaf_node", "path_q_len",
              "q_offsets", "q", "out"):
        setattr(d, n, OK)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_ROWS = [(dict(struct_size=8), B.SS_ERR_INVALID_ARG), (dict(flags=2), B.SS_ERR_INVALID_ARG), (dict(n_rows=-1), B.SS_ERR_INVALID_ARG),
            (dict(num_q_heads=0), B.SS_ERR_INVALID_ARG), (dict(num_kv_heads=-1), B.SS_ERR_INVALID_ARG), (dict(eps=-1.0), B.SS_ERR_INVALID_ARG),
            (dict(eps=float("nan")), B.SS_ERR_INVALID_ARG), (dict(inv_freq=None), B.SS_ERR_INVALID_ARG), (dict(q_out=None), B.SS_ERR_INVALID_ARG),
            (dict(q=None), B.SS_ERR_INVALID_ARG), (dict(head_dim=64), B.SS_ERR_UNSUPPORTED), (dict(rot_dim=24), B.SS_ERR_UNSUPPORTED),
            (dict(rot_dim=144), B.SS_ERR_UNSUPPORTED), (dict(rot_dim=-16), B.SS_ERR_INVALID_ARG), (dict(q=OK + 8), B.SS_ERR_UNSUPPORTED),
            (dict(k_weight=OK + 2), B.SS_ERR_UNSUPPORTED), (dict(k_row_stride=2044), B.SS_ERR_UNSUPPORTED),
            (dict(v_head_stride=4), B.SS_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("kw,rc", BAD_ROWS)
def test_rows_are_checked(lib, kw, rc):
    r = rows(k_out=OK, **kw)
    assert lib.ss_qk_norm_rope(ctypes.byref(r), None) == rc
    r = rows(v=OK, **kw)
    assert lib.ss_kv_append(ctypes.byref(desc()), ctypes.byref(r), None) == rc


def test_norm_rope_arguments(lib):
    call = lambda **kw: lib.ss_qk_norm_rope(ctypes.byref(rows(**kw)), None)
    assert lib.ss_qk_norm_rope(None, None) == B.SS_ERR_INVALID_ARG
    assert call() == B.SS_ERR_INVALID_ARG                                  # keys without a place to go
    assert call(k=None, k_out=OK) == B.SS_ERR_INVALID_ARG
    assert call(k=None, q=None, q_out=None) == B.SS_ERR_INVALID_ARG
    assert call(k_out=OK, positions=None) == B.SS_ERR_INVALID_ARG
    assert call(k_out=OK, n_rows=0) == B.SS_OK


@pytest.mark.parametrize("kw,rc", [
    (dict(struct_size=8), B.SS_ERR_INVALID_ARG), (dict(num_paths=-1), B.SS_ERR_INVALID_ARG), (dict(head_dim=64), B.SS_ERR_UNSUPPORTED),
    (dict(page_size=32), B.SS_ERR_UNSUPPORTED), (dict(kv_token_stride=256), B.SS_ERR_UNSUPPORTED),
    (dict(kv_head_stride=64), B.SS_ERR_UNSUPPORTED), (dict(kv_page_stride=0), B.SS_ERR_UNSUPPORTED),
    (dict(num_kv_heads=4), B.SS_ERR_INVALID_ARG), (dict(num_q_heads=14), B.SS_ERR_INVALID_ARG), (dict(k_pool=None), B.SS_ERR_INVALID_ARG),
    (dict(v_pool=OK + 16), B.SS_ERR_UNSUPPORTED), (dict(q_offsets=None), B.SS_ERR_INVALID_ARG), (dict(num_paths=0), B.SS_OK),
    (dict(total_q=0), B.SS_OK)])
def test_append_descriptor(lib, kw, rc):
    assert lib.ss_kv_append(ctypes.byref(desc(**kw)), ctypes.byref(rows(v=OK)), None) == rc


def test_append_arguments(lib):
    call = lambda **kw: lib.ss_kv_append(ctypes.byref(desc()), ctypes.byref(rows(**kw)), None)
    assert lib.ss_kv_append(None, ctypes.byref(rows(v=OK)), None) == B.SS_ERR_INVALID_ARG
    assert lib.ss_kv_append(ctypes.byref(desc()), None, None) == B.SS_ERR_INVALID_ARG
    assert call() == B.SS_ERR_INVALID_ARG                                  # no values
    assert call(v=OK, k=None) == B.SS_ERR_INVALID_ARG
    assert call(v=OK, k_out=OK) == B.SS_ERR_INVALID_ARG
    assert call(v=OK, n_rows=0) == B.SS_OK


@pytest.mark.parametrize("kw,rc", [
    (dict(struct_size=8), B.SS_ERR_INVALID_ARG), (dict(flags=0x100), B.SS_ERR_INVALID_ARG), (dict(num_q_heads=13), B.SS_ERR_UNSUPPORTED),
    (dict(num_q_heads=0), B.SS_ERR_INVALID_ARG), (dict(num_q_heads=258), B.SS_ERR_UNSUPPORTED), (dict(page_size=8), B.SS_ERR_UNSUPPORTED),
    (dict(sm_scale=-1.0), B.SS_ERR_INVALID_ARG), (dict(sm_scale=float("inf")), B.SS_ERR_INVALID_ARG),
    (dict(total_q=1 << 40), B.SS_ERR_UNSUPPORTED), (dict(q_src_offsets=OK, q_src_rows=-1), B.SS_ERR_INVALID_ARG),
    (dict(max_sms=-1), B.SS_ERR_INVALID_ARG)])
def test_draft_descriptor(lib, kw, rc):
    out = ctypes.c_size_t(0)
    assert lib.ss_draft_attention_workspace_bytes(ctypes.byref(desc(**kw)), ctypes.byref(out)) == rc
    assert lib.ss_draft_attention(ctypes.byref(desc(**kw)), OK, OK, 1 << 40, None) == rc


def test_draft_arguments(lib):
    call = lambda ws=OK, nbytes=1 << 40, **kw: lib.ss_draft_attention(ctypes.byref(desc(**kw)), OK, ws, nbytes, None)
    assert call(ws=None) == B.SS_ERR_INVALID_ARG
    assert call(ws=OK + 64) == B.SS_ERR_INVALID_ARG
    assert call(q=None) == B.SS_ERR_INVALID_ARG
    assert call(path_q_len=None) == B.SS_ERR_INVALID_ARG
    assert call(out=OK + 16) == B.SS_ERR_UNSUPPORTED
    assert call(q=OK + 8) == B.SS_ERR_UNSUPPORTED
    assert call(k_pool=OK + 128) == B.SS_ERR_UNSUPPORTED
    size = B.ss_draft_attention_workspace_bytes(desc())
    assert size % 256 == 0 and call(nbytes=size - 1) == B.SS_ERR_WORKSPACE_TOO_SMALL
    assert B.ss_draft_attention_workspace_bytes(desc(num_paths=5000, total_q=70000)) > size
    assert lib.ss_draft_attention_workspace_bytes(ctypes.byref(desc()), None) == B.SS_ERR_INVALID_ARG


def sample(**kw):
    d = B.ss_sample_desc_t()
    d.struct_size = ctypes.sizeof(B.ss_sample_desc_t)
    d.n_seq, d.vocab, d.row_stride, d.temperature_all, d.top_p_all = 4, 1000, 1000, 1.0, 1.0
    d.logits = d.draw_offsets = d.uniforms = d.tokens_out = OK
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw,rc", [
    (dict(struct_size=4), B.SS_ERR_INVALID_ARG), (dict(flags=1), B.SS_ERR_INVALID_ARG), (dict(n_seq=-1), B.SS_ERR_INVALID_ARG),
    (dict(vocab=0), B.SS_ERR_INVALID_ARG), (dict(row_stride=999), B.SS_ERR_INVALID_ARG), (dict(logits_type=2), B.SS_ERR_INVALID_ARG),
    (dict(vocab=2097153, row_stride=2097153), B.SS_ERR_UNSUPPORTED)])
def test_sample_descriptor(lib, kw, rc):
    out = ctypes.c_size_t(0)
    assert lib.ss_filtered_sample_workspace_bytes(ctypes.byref(sample(**kw)), ctypes.byref(out)) == rc
    assert lib.ss_filtered_sample(ctypes.byref(sample(**kw)), OK, 1 << 40, None) == rc


def test_sample_arguments(lib):
    call = lambda ws=OK, nbytes=1 << 40, **kw: lib.ss_filtered_sample(ctypes.byref(sample(**kw)), ws, nbytes, None)
    assert call(ws=None) == B.SS_ERR_INVALID_ARG
    assert call(ws=OK + 16) == B.SS_ERR_INVALID_ARG
    assert call(logits=None) == B.SS_ERR_INVALID_ARG
    assert call(draw_offsets=None) == B.SS_ERR_INVALID_ARG
    assert call(logits=OK + 2) == B.SS_ERR_UNSUPPORTED
    assert call(n_seq=0, logits=None) == B.SS_OK
    size = B.ss_filtered_sample_workspace_bytes(sample())
    assert size % 256 == 0 and call(nbytes=size - 1) == B.SS_ERR_WORKSPACE_TOO_SMALL
    assert lib.ss_filtered_sample_workspace_bytes(ctypes.byref(sample()), None) == B.SS_ERR_INVALID_ARG


def test_a_call_runs_on_the_device_of_its_tensors(monkeypatch):
    at, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, at[0] = at[0], self.index

        def __exit__(self, *a):
            at[0] = self.before

    monkeypatch.setattr(B.torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(B.torch.cuda, "device", Device)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 40 + device)
    call = lambda *a: seen.append((at[0],) + a) or B.SS_OK
    for device, stream in ((None, None), (0, None), (2, None), (2, 7)):
        B._call(device, call, "x", stream=stream)
    assert seen == [(0, "x", 40), (0, "x", 40), (2, "x", 42), (2, "x", 7)] and at[0] == 0
