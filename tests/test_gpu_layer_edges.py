"""Layer norm, 16-bit linears and 8-bit activations at values where they can go wrong: infinities and NaN, GELU's tail, subnormal scales, ties."""
import math

import pytest
import torch

import layer_reference as ref
import test_gpu_layer_norm as layer_norm

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("W,eps", [(1, 1e-12), (40, 0.0), (100, 1e-12), (200, 0.0), (500, 1e-12), (1000, 0.0), (1500, 1e-12), (3001, 0.0), (8200, 1e-12), (20000, 0.0)])
def test_norm_rows_that_are_no_numbers(qb, t, W, eps):
    """NaN and infinities of a row reach all of its Y, mean, rstd, codes and dX, dweight and dbias as the formulas say, and no other row"""
    X = ref.draw(7, W, seed=W, t=t, mean=0.3)
    w, dY = ref.draw(W, seed=1, mean=1.0, std=0.2, t=torch.float32).cuda(), ref.draw(7, W, seed=2, t=t).cuda()
    clean = qb.qb_layer_norm_fwd(X.cuda(), w, eps=eps, keep=True)
    clean_dX = qb.qb_layer_norm_bwd(dY, X.cuda(), w, clean[1], clean[2])[0]
    X[1, W // 2], X[2, W - 1], X[4, 0], X[5, 0], X[5, W - 1] = math.nan, math.inf, -math.inf, math.inf, -math.inf
    Y, mean, rstd, codes, scales = qb.qb_layer_norm_fwd(X.cuda(), w, eps=eps, keep=True)
    dX, dw, db = qb.qb_layer_norm_bwd(dY, X.cuda(), w, mean, rstd)
    good, bad = [0, 3, 6], [1, 2, 4, 5]
    for got, want in zip((Y, mean, rstd, codes, scales, dX), (*clean, clean_dX)):
        assert torch.equal(got[good], want[good])
    assert torch.equal(mean.cpu().nan_to_num(nan=7.0)[bad], X.double().mean(1).float().nan_to_num(nan=7.0)[bad])  # NaN, the infinities, NaN (one value: that value)
    assert rstd[bad].isnan().all() and Y[bad].isnan().all() and dX[bad].isnan().all()
    assert qb.qb_restore_act(codes, scales, torch.float32)[bad].isnan().all()
    assert dw.isnan().all() and db.isfinite().all()


def tail_off(z):
    """what the kernels' normal distribution is off, relative to its smaller tail: fitted up to 7; further out it falls faster than the true one"""
    return torch.where(z.abs() <= 7, ref.NORMAL, torch.where(z.abs() <= 9, 0.02, 1.0))


def from_minus_to_plus(T, t):
    """[T, 64] values of `t` from -16 to 16, most of them between -9 and 9"""
    z = torch.cat([torch.linspace(-9, 9, T * 64 - 64, dtype=torch.float64), torch.linspace(-16, 16, 64, dtype=torch.float64)])
    return z[torch.randperm(T * 64, generator=torch.Generator().manual_seed(T))].view(T, 64).to(t)


FLUSHED = 2.0 ** -126  # the hardware's power of two has no subnormal results: below this it is zero


def rounded(t, value):
    return ref.half_step(t) * value.abs() * (1 + 2 * ref.half_step(t)) + torch.finfo(t).tiny * torch.finfo(t).eps


@pytest.mark.parametrize("t", TYPES[1:])
@pytest.mark.parametrize("T", [40, 700, 9000])
def test_gelu_derivative_and_its_tail(qb, t, T):
    """dX of a layer whose product is one, so that what is left is the derivative at each value: relative to its two terms, however small"""
    pre = from_minus_to_plus(T, t)
    dY, W = torch.zeros(T, 8, dtype=t), torch.zeros(8, 64, dtype=t)
    dY[:, 3] = W[3] = 1
    dX = qb.qb_linear_bwd(dY.cuda(), None, W.cuda(), pre=pre.cuda(), act="gelu", need=(True, False, False))[0]
    z = pre.double()
    bell, tail = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), ref.phi(-z.abs())
    want = ref.phi(z) + z * bell
    # the exponent is rounded three times, to half a step each, and so is relative 1.5 z^2 half steps off; the exponential, the products and the last sum have eight between
    # them; right of zero the sum is of the order of one, with two of its own
    # (and where the exponential is below the normal numbers, at 13 and beyond, it is zero)
    off = (1 + z.abs()) * FLUSHED + tail_off(z) * tail + (1.5 * z * z + 8) * ref.STEP * z.abs() * bell + 2 * ref.STEP * torch.where(z < 0, 0.0, 1.0 + z.abs() * bell)
    ref.near(dX, want, rounded(t, want) + off, "GELU's derivative")


@pytest.mark.parametrize("t", TYPES[1:])
@pytest.mark.parametrize("T,N", [(40, 8), (700, 8), (9000, 8), (2000, 520)])
def test_gelu_and_its_tail(qb, t, T, N):
    """GELU at values that are known exactly: relative to itself, however small"""
    z = from_minus_to_plus(T, t)[:, 0].contiguous()
    X, W = torch.zeros(T, 64, dtype=t), torch.zeros(N, 64, dtype=t)
    X[:, 5], W[:, 5] = z, 1
    Y = qb.qb_linear_fwd(X.cuda(), W.cuda(), act="gelu")
    z = z.double()[:, None].expand(T, N)
    want = z * ref.phi(z)
    off = z.abs() * (FLUSHED + tail_off(z) * ref.phi(-z.abs()) + 2 * ref.STEP * torch.where(z < 0, ref.phi(z), 1.0))
    ref.near(Y, want, rounded(t, want) + off, "GELU")


def test_codes_of_subnormal_scales(qb):
    """every multiple of the least subnormal number over scales of 1 to 41 of them: quotients next to half a step, whose distance from it is less than a subnormal step"""
    for n in range(1, 42):
        k = torch.arange(127 * n + 1, dtype=torch.int32)
        k = torch.cat([k, k.new_zeros(-len(k) % 63)]).view(-1, 63)
        k = torch.cat([torch.full((len(k), 1), 127 * n, dtype=torch.int32), k], 1)
        x = k.view(torch.float32) * torch.where(torch.arange(64) % 3 == 1, -1.0, 1.0)
        codes, scales = qb.qb_checkpoint_act(x.cuda())
        assert (scales.cpu().view(torch.int32) == n).all()
        # a quotient of whole numbers, rounded half to even in whole numbers
        low, rest = k // n, 2 * (k % n)
        want = (low + ((rest > n) | ((rest == n) & (low % 2 == 1))).int()) * torch.where(torch.arange(64) % 3 == 1, -1, 1)
        assert torch.equal(codes.cpu().int(), want)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,W", [(131, 8193), (300, 8256), (131, 10000), (3, 20001), (140, 32768)])
def test_norm_sums_of_wide_rows_from_8_bits(qb, t, T, W):
    """rows that are read a second time for the sums over the tokens, in 8 bits"""
    layer_norm.test_backward_from_8_bits(qb, t, T, W)
