"""Refusals at the edges of the operators' interface, before a launch (no GPU needed)."""
import pytest

import paper_1909_05840_amd as qb
from test_operators_host import AT16, P, WORKSPACE, attention, grads


@pytest.fixture(scope="module")
def lib():
    return qb.load_library()


@pytest.mark.parametrize("workspace", [None, AT16])
def test_keys_without_queries_need_the_workspace_too(lib, workspace):
    """max_q is an upper bound: with none in the tensor the first launch still writes its statistics' last entries"""
    a = attention(total_q=0, Q=None)
    assert lib.qb_attention_bwd_workspace_nbytes(a) > 0
    assert lib.qb_attention_bwd(a, None, None, None, grads(dQ=None), workspace, None) == WORKSPACE
    assert lib.qb_attention_bwd(a, P, P, P, grads(), workspace, None) == WORKSPACE
