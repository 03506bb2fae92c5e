"""The 16-bit linears' backward where its first launch has more work than a launch has threads: 2^36 values of X, or of dY."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu
T = 1 << 24
BF16 = torch.bfloat16


@pytest.fixture
def room():
    """free memory in GB"""
    torch.cuda.empty_cache()
    yield torch.cuda.mem_get_info()[0] / 1e9
    torch.cuda.empty_cache()


def tokens():
    """Tokens whose dY is not zero: the first and the last ones, and some between; with 2^36 values a first launch of the most threads ends 64 to 512 rows before the last."""
    g = torch.Generator().manual_seed(1)
    return torch.cat([torch.arange(8), torch.randint(8, T - 2000, (300,), generator=g), torch.arange(T - 2000, T)]).unique().cuda()


def test_input_from_8_bits(qb, room):
    N, K = 8, 4160
    assert T * K > 1 << 36
    if room < 235:
        pytest.skip("the codes, and the values in 16 bits that they stand for, are 215 GB")
    codes, scales = torch.empty(T, K, dtype=torch.int8, device="cuda"), torch.empty(T, K // 64, device="cuda")
    for at in range(0, T, 1 << 20):  # (rows that differ from each other, in one pass over each)
        codes[at:at + (1 << 20)].random_(-127, 128)
    scales.uniform_(0.5, 1.5)
    dY, at = torch.zeros(T, N, dtype=BF16, device="cuda"), tokens()
    dY[at] = ref.draw(len(at), N, seed=2, t=BF16).cuda()
    W = torch.zeros(N, K, dtype=BF16, device="cuda")
    dW = qb.qb_linear_bwd(dY, (codes, scales), W, need=(False, True, False))[1].double()
    x = qb.qb_restore_act(codes[at], scales[at], BF16).double()
    d = dY[at].double()
    want, size = d.T @ x, d.abs().T @ x.abs()
    # sums of as many numbers as there are tokens with a gradient (zeros add nothing), binary32 in any order
    assert ((dW - want).abs() <= ref.half_step(BF16) * want.abs() * 1.01 + (len(at) + 2) * ref.STEP * size).all()


def test_gradients_that_are_copied(qb, room):
    """dY is one row for all tokens, which is no multiple of sixteen bytes: its copy has 2^36 values"""
    N, K = 4153, 64
    assert T * (N + 7) > 1 << 36
    if room < 160:
        pytest.skip("dY's copy is 140 GB")
    d, W = ref.draw(1, N, seed=3, t=BF16).cuda(), ref.draw(N, K, seed=4, std=N ** -0.5, t=BF16).cuda()
    dX = qb.qb_linear_bwd(d.expand(T, N), None, W, need=(True, False, False))[0]
    one = d.double() @ W.double()
    size = d.double().abs() @ W.double().abs()
    assert ((dX[:1].double() - one).abs() <= ref.half_step(BF16) * one.abs() * 1.01 + (N + 2) * ref.STEP * size).all()
    assert torch.equal(dX, dX[:1].expand(T, K))  # (a row's sums are formed in the same order, whatever the row)
