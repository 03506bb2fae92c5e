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


@pytest.mark.parametrize("scale,fine", [(9e-37, False), (1e-38, False), (1.1e-36, True), (1.9e8, True), (2.1e8, False), (1e38, False)])
def test_scales_that_binary32_has_no_room_for(lib, scale, fine):
    """lse / scale of a row, and the maximum before a row has seen a key times scale, have to be finite numbers"""
    a = attention(scale=scale, total_q=0, total_k=0)  # (nothing to do where it is taken)
    want = 0 if fine else 7
    assert lib.qb_attention_fwd(a, P, P, P, None) == want
    assert lib.qb_attention_bwd(a, P, P, P, grads(), P, None) == want
