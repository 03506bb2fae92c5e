"""The 16-bit linears against 64 bits in calls that between them take every kernel, with the epilogues and the inputs that these kernels have."""
import pytest
import torch

import test_gpu_linear16 as linear16
from linear_plans import BACKWARD, FORWARD, NEEDS
from test_gpu_linear16 import check_backward, check_forward

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,N,K", FORWARD)
def test_forward(qb, t, T, N, K):
    check_forward(qb, T, N, K, t, act="gelu", residual=True, keep="codes")
    check_forward(qb, T, N, K, t, act="tanh", keep="values", wide=True)
    check_forward(qb, T, N, K, t, keep="codes", bias=False, residual=True, wide=True)
    check_forward(qb, T, N, K, t, act="relu")


@pytest.mark.parametrize("T,N,K", BACKWARD)
def test_backward(qb, T, N, K):
    t = TYPES[(T + N) % 2]
    for need in NEEDS:
        check_backward(qb, T, N, K, t, need=need)
    # the derivative in front, its input formed again; gradients and tokens in rows apart, which are copied where they are no multiple of sixteen bytes
    check_backward(qb, T, N, K, t, x="again", pre="codes", act="gelu")
    check_backward(qb, T, N, K, TYPES[(T + N + 1) % 2], x="given", pre="values", act="tanh", wide=3)
    check_backward(qb, T, N, K, t, x="again", pre="values", act="relu", need=(True, False, True))
    check_backward(qb, T, N, K, t, x="codes", need=(False, True, True), wide=8)


@pytest.mark.parametrize("T,N,K", [(8237, 1, 4288), (71, 8521, 2560), (24, 3315, 2048), (6991, 68, 3200), (2281, 6711, 64), (6178, 2131, 128), (6897, 4375, 192), (8190, 1024, 1024)])
def test_workspaces_of_exactly_the_size(qb, T, N, K):
    """parts of small, middle and large tiles, and the copies of dY and X beside them"""
    linear16.test_workspaces_of_exactly_the_size(qb, T, N, K)
