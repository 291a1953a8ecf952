"""Sizes whose indices would pass 32 bits are refused: nothing is launched and no pointer is followed.  (No device holds
such a node, but its pages may be named many times over.)"""
import pytest

from paper_2609_39334_b200 import binding as B
from test_long_search_operators_cpu import evict, key_weights, lib, nothing_launched, run_evict, run_weights  # noqa: F401
from test_step_operators_cpu import OK, desc

U = B.SS_ERR_UNSUPPORTED


# Nodes of so many pages end less than two tiles of 128 keys in front of 2^31 (the loops' next key would not fit), or behind it.
@pytest.mark.parametrize("pages", [0x7ffffff - 14, 0x7ffffff, 0x8000000])
def test_key_weights_refuses_nodes_that_end_at_two_to_the_31(lib, pages):  # noqa: F811
    assert run_weights(lib, desc(lse=OK, total_node_pages=pages), key_weights()) == (U, U)


@pytest.mark.parametrize("what", ["num_nodes", "num_paths"])
def test_key_weights_refuses_so_many_nodes_or_paths(lib, what):  # noqa: F811
    """(The planner's threads step by 8192 of them.)"""
    for n in (0x7fffffff, 0x40000001):
        assert run_weights(lib, desc(lse=OK, **{what: n}), key_weights()) == (U, U)


def test_key_weights_takes_what_is_just_shorter(lib):  # noqa: F811
    d = desc(lse=OK, total_node_pages=0x7ffffff - 15)
    assert B.ss_key_weights_workspace_bytes(d, key_weights()) > 0


# (A block's threads look four quads of slots ahead, 8192 slots.)
@pytest.mark.parametrize("pages", [0x7ffffff - 1022, 0x7ffffff, 0x8000000])
def test_evict_refuses_nodes_that_end_at_two_to_the_31(lib, pages):  # noqa: F811
    assert run_evict(lib, desc(total_node_pages=pages), evict()) == (U, U)


def test_evict_takes_what_is_just_shorter(lib):  # noqa: F811
    assert B.ss_kv_evict_workspace_bytes(desc(total_node_pages=0x7ffffff - 1023), evict()) > 0
