"""Layer norm, 16-bit linears and 8-bit activations at values where they can go wrong: infinities and NaN, GELU's tail, subnormal scales, ties."""
import math

import pytest
import torch

import layer_reference as ref

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
