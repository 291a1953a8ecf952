"""Refusals of the operators of long searches on the host - weights of keys, eviction, axes, rules on logits: nothing is launched and no
pointer is followed."""
import ctypes

import pytest
import torch

from paper_2609_39334_b200 import binding as B
from paper_2609_39334_b200 import build as cuda_build
from test_operator_bindings_cpu import Claimed
from test_step_operators_cpu import OK, desc, rows

BIG = 1 << 40
INF, NAN = float("inf"), float("nan")
A, U, W = B.SS_ERR_INVALID_ARG, B.SS_ERR_UNSUPPORTED, B.SS_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return B.lib()


@pytest.fixture(autouse=True)
def nothing_launched(lib):
    before = B.ss_launch_count()
    yield
    assert B.ss_launch_count() == before


def filled(kind, given, **kw):
    s = kind()
    s.struct_size = ctypes.sizeof(kind)
    for k, v in {**given, **kw}.items():
        setattr(s, k, v)
    return s


def axes(**kw):
    return filled(B.ss_axes_t, dict(num_axes=3, position_stride=10, positions=OK, pair_axis=OK), **kw)


def key_weights(**kw):
    return filled(B.ss_key_weights_t, dict(decay=1.0, weights_in=OK, weights_out=OK, order=OK, path_order=OK), **kw)


def evict(**kw):
    return filled(B.ss_evict_t, dict(n_nodes=4, nodes=OK, keep=OK, weights=OK, kv_len_out=OK), **kw)


def rules(**kw):
    return filled(B.ss_logit_rules_t, dict(n_seq=4, vocab=1000, logits_type=B.SS_LOGITS_FP32, row_stride=1000, out_row_stride=1000, mask_stride=32,
                                           repetition_all=1.0, logits=OK, out=2 * OK, history=OK, history_offsets=OK, prompts=OK, prompt_offsets=OK,
                                           n_prompts=1, bias_tokens=OK, bias_values=OK, bias_offsets=OK, n_biases=1, masks=OK, n_masks=1), **kw)


@pytest.mark.parametrize("kw,rc", [
    (dict(struct_size=8), A), (dict(num_axes=0), A), (dict(num_axes=5), U), (dict(position_stride=-1), A), (dict(position_stride=9), A),
    (dict(positions=None), A), (dict(pair_axis=None), A)])
def test_axes(lib, kw, rc):
    r, a = rows(positions=None, k=None), axes(**kw)
    assert lib.ss_qk_norm_rope_axes(ctypes.byref(r), ctypes.byref(a), None) == rc
    r = rows(positions=None, v=OK)
    assert lib.ss_kv_append_axes(ctypes.byref(desc()), ctypes.byref(r), ctypes.byref(a), None) == rc


def test_axes_and_positions_or_none(lib):
    a = axes()
    assert lib.ss_qk_norm_rope_axes(ctypes.byref(rows(k=None)), ctypes.byref(a), None) == A
    assert lib.ss_kv_append_axes(ctypes.byref(desc()), ctypes.byref(rows(v=OK)), ctypes.byref(a), None) == A
    assert lib.ss_qk_norm_rope_axes(ctypes.byref(rows(k=None, positions=None)), None, None) == A
    assert lib.ss_qk_norm_rope_axes(ctypes.byref(rows(k=None, positions=None, n_rows=0)), ctypes.byref(a), None) == B.SS_OK
    assert lib.ss_qk_norm_rope_axes(ctypes.byref(rows(k=None, positions=None, head_dim=64)), ctypes.byref(a), None) == U


BAD_DESC = [(dict(struct_size=8), A), (dict(num_kv_heads=0), A), (dict(head_dim=64), U), (dict(page_size=32), U), (dict(kv_token_stride=256), U),
            (dict(kv_page_stride=100), U), (dict(kv_head_stride=0), U), (dict(num_nodes=-1), A), (dict(num_pages=-1), A), (dict(total_node_pages=-1), A),
            (dict(total_node_pages=1 << 28), U)]


def run_weights(lib, d, k, ws=OK, size=BIG):
    out = ctypes.c_size_t(0)
    sized = lib.ss_key_weights_workspace_bytes(ctypes.byref(d), ctypes.byref(k), ctypes.byref(out))
    return sized, lib.ss_key_weights(ctypes.byref(d), ctypes.byref(k), ws, size, None)


@pytest.mark.parametrize("kw,rc", BAD_DESC + [(dict(num_q_heads=13), U), (dict(num_q_heads=2 * 129), U), (dict(sm_scale=-1.0), A), (dict(sm_scale=INF), A),
                                              (dict(flags=1 << 9), A), (dict(max_sms=-1), A), (dict(total_q=-1), A), (dict(total_q=1 << 28), U)])
def test_key_weights_descriptor(lib, kw, rc):
    assert run_weights(lib, desc(lse=OK, **kw), key_weights()) == (rc, rc)


@pytest.mark.parametrize("kw,rc", [(dict(struct_size=8), A), (dict(flags=1), A), (dict(decay=-0.5), A), (dict(decay=NAN), A), (dict(decay=INF), A),
                                   (dict(last_tokens=-1), A)])
def test_key_weights_arguments(lib, kw, rc):
    assert run_weights(lib, desc(lse=OK), key_weights(**kw)) == (rc, rc)


def test_key_weights_pointers(lib):
    for kw in (dict(weights_out=None),):
        assert run_weights(lib, desc(lse=OK), key_weights(**kw)) == (B.SS_OK, A)
    for kw in (dict(weights_out=OK + 4), dict(weights_in=OK + 32), dict(order=OK + 16)):
        assert run_weights(lib, desc(lse=OK), key_weights(**kw)) == (B.SS_OK, U)
    for kw in (dict(lse=None), dict(q=None), dict(k_pool=None), dict(node_pages=None), dict(path_q_len=None), dict(node_parent=None)):
        assert run_weights(lib, desc(**{"lse": OK, **kw}), key_weights()) == (B.SS_OK, A)
    for kw in (dict(k_pool=OK + 128), dict(q=OK + 8)):
        assert run_weights(lib, desc(lse=OK, **kw), key_weights()) == (B.SS_OK, U)
    assert run_weights(lib, desc(lse=OK), key_weights(), ws=None) == (B.SS_OK, A)
    assert run_weights(lib, desc(lse=OK), key_weights(), ws=OK + 8) == (B.SS_OK, A)
    assert run_weights(lib, desc(lse=OK), key_weights(), size=1000) == (B.SS_OK, W)
    assert lib.ss_key_weights_workspace_bytes(ctypes.byref(desc()), None, ctypes.byref(ctypes.c_size_t())) == A


def run_evict(lib, d, e, ws=OK, size=BIG):
    out = ctypes.c_size_t(0)
    sized = lib.ss_kv_evict_workspace_bytes(ctypes.byref(d), ctypes.byref(e), ctypes.byref(out))
    return sized, lib.ss_kv_evict(ctypes.byref(d), ctypes.byref(e), ws, size, None)


@pytest.mark.parametrize("kw,rc", BAD_DESC)
def test_evict_descriptor(lib, kw, rc):
    assert run_evict(lib, desc(**kw), evict()) == (rc, rc)


@pytest.mark.parametrize("kw,rc", [(dict(struct_size=8), A), (dict(flags=1), A), (dict(n_nodes=-1), A), (dict(max_keys=-1), A), (dict(sinks=-1), A),
                                   (dict(recent=-1), A), (dict(n_nodes=0x7fffffff), U)])
def test_evict_arguments(lib, kw, rc):
    assert run_evict(lib, desc(), evict(**kw)) == (rc, rc)


def test_evict_pointers(lib):
    for kw in (dict(nodes=None), dict(keep=None), dict(weights=None)):
        assert run_evict(lib, desc(), evict(**kw)) == (B.SS_OK, A)
    for kw in (dict(k_pool=None), dict(v_pool=None), dict(node_kv_len=None), dict(node_page_offsets=None), dict(node_pages=None)):
        assert run_evict(lib, desc(**kw), evict()) == (B.SS_OK, A)
    assert run_evict(lib, desc(v_pool=OK + 64), evict()) == (B.SS_OK, U)
    assert run_evict(lib, desc(), evict(), ws=None) == (B.SS_OK, A)
    assert run_evict(lib, desc(), evict(), ws=OK + 128) == (B.SS_OK, A)
    assert run_evict(lib, desc(), evict(), size=512) == (B.SS_OK, W)


@pytest.mark.parametrize("kw,rc", [
    (dict(struct_size=8), A), (dict(flags=1), A), (dict(n_seq=-1), A), (dict(vocab=-1), A), (dict(logits_type=2), A), (dict(row_stride=999), A),
    (dict(out_row_stride=999), A), (dict(vocab=2097153, row_stride=BIG, out_row_stride=BIG, mask_stride=BIG), U), (dict(logits=None), A), (dict(out=None), A),
    (dict(out=OK, out_row_stride=1001), A), (dict(logits=OK + 2), A), (dict(out=OK + 1, logits_type=B.SS_LOGITS_BF16), A), (dict(history_offsets=None), A),
    (dict(prompt_offsets=None), A), (dict(bias_offsets=None), A), (dict(bias_values=None), A), (dict(bias_tokens=None), A), (dict(mask_stride=31), A),
    (dict(n_prompts=-1), A), (dict(n_biases=-1), A), (dict(n_masks=-1), A), (dict(n_seq=0x7fffffff, vocab=100000, row_stride=100000, out_row_stride=100000, mask_stride=4000), U)])
def test_rules(lib, kw, rc):
    assert lib.ss_logit_rules(ctypes.byref(rules(**kw)), None) == rc


def test_rules_without_work(lib):
    assert lib.ss_logit_rules(ctypes.byref(rules(n_seq=0, logits=None, out=None)), None) == B.SS_OK
    assert lib.ss_logit_rules(ctypes.byref(rules(vocab=0)), None) == B.SS_OK
    assert lib.ss_logit_rules(None, None) == A


def test_bindings_refuse_what_would_be_read_out_of_bounds(lib):
    i32, f32 = (lambda *s: Claimed(torch.zeros(*s, dtype=torch.int32))), (lambda *s: Claimed(torch.zeros(*s)))
    kw = B.make_key_weights(weights_out=f32(99, 2, 16))
    with pytest.raises(AssertionError):                           # fewer pages than the pool
        B.ss_key_weights(desc(lse=OK), kw, torch.zeros(256, dtype=torch.uint8))
    kw = B.make_key_weights(weights_out=f32(100, 2, 16), path_order=i32(7))
    with pytest.raises(AssertionError):                           # fewer than the paths
        B.ss_key_weights(desc(lse=OK), kw, torch.zeros(256, dtype=torch.uint8))
    ev = B.make_evict(nodes=i32(3), keep=i32(3), weights=f32(100, 2, 16), order=i32(90, 2, 16))
    with pytest.raises(AssertionError):
        B.ss_kv_evict(desc(), ev, torch.zeros(256, dtype=torch.uint8))
    for make in (lambda: B.make_evict(nodes=i32(3), keep=i32(2), weights=f32(100, 2, 16)),
                 lambda: B.make_key_weights(weights_out=f32(100, 32)),
                 lambda: B.make_key_weights(weights_out=i32(100, 2, 16)),
                 lambda: B.make_logit_rules(logits=f32(4, 100), out=f32(4, 101)),
                 lambda: B.make_logit_rules(logits=f32(4, 100), history=i32(9)),
                 lambda: B.make_logit_rules(logits=f32(4, 100), history=i32(9), history_offsets=Claimed(torch.zeros(4, dtype=torch.int64))),
                 lambda: B.make_logit_rules(logits=f32(4, 100), masks=i32(4, 3)),
                 lambda: B.make_logit_rules(logits=f32(4, 100), repetition=f32(3)),
                 lambda: B.make_axes(positions=i32(3, 10), pair_axis=f32(64))):
        with pytest.raises((AssertionError, AttributeError)):
            make()
    r = rows(positions=None, k=None)
    with pytest.raises(AssertionError):                           # fewer positions than rows
        B.ss_qk_norm_rope_axes(r, B.make_axes(positions=i32(3, 9), pair_axis=i32(64)))
