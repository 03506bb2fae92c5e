"""Layer norm, 16-bit linears and 8-bit activations where offsets pass 32 bits: more than 2^32 values, rows around 2^31, 2^32 and the end looked at."""
import pytest
import torch

import layer_reference as ref
from layer_reference import STEP, half_step

pytestmark = pytest.mark.gpu
T = (1 << 20) + 3
BF16 = torch.bfloat16


def values(rows, columns, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(rows, columns, device="cuda", dtype=BF16, generator=g)


def places(width):
    """first rows of three stretches: at 2^31 and 2^32 values, and the last one"""
    return [(1 << 31) // width - 20, min((1 << 32) // width - 20, T - 40), T - 40]


def within(got, want, off, what):
    bad = ~((got.double() - want).abs() <= off)
    assert not bad.any(), "%s: %d of %d outside" % (what, int(bad.sum()), bad.numel())


@pytest.mark.parametrize("W", [4096, 4100])
def test_rows_of_their_own(qb, W):
    """a row's results are those of a call that has few rows"""
    X, dY = values(T, W, 1), values(T, W, 2)
    assert X.numel() > 1 << 32
    codes, scales = qb.qb_checkpoint_act(X)
    back = qb.qb_restore_act(codes, scales, BF16)
    for at in places(W):
        few = qb.qb_checkpoint_act(X[at:at + 40])
        assert torch.equal(codes[at:at + 40], few[0]) and torch.equal(scales[at:at + 40], few[1])
        assert torch.equal(back[at:at + 40], qb.qb_restore_act(*few, BF16))
    del back
    w = torch.linspace(0.5, 1.5, W, device="cuda")
    Y, mean, rstd, c8, s8 = qb.qb_layer_norm_fwd(X, w, keep=True)
    dX = qb.qb_layer_norm_bwd(dY, (codes, scales), w, mean, rstd, residual=X)[0]
    for at in places(W):
        part = slice(at, at + 40)
        few = qb.qb_layer_norm_fwd(X[part], w, keep=True)
        assert all(torch.equal(a[part], b) for a, b in zip((Y, mean, rstd, c8, s8), few))
        assert torch.equal(dX[part], qb.qb_layer_norm_bwd(dY[part], (codes[part], scales[part]), w, mean[part], rstd[part], residual=X[part])[0])


@pytest.mark.parametrize("N,K", [(4097, 64), (64, 4160)])
def test_linear(qb, N, K):
    t = BF16
    X, dY, W = values(T, K, 1), values(T, N, 2), ref.draw(N, K, seed=3, std=K ** -0.5, t=t).cuda()
    w = W.double()
    Y = qb.qb_linear_fwd(X, W)
    for at in places(max(N, K)):
        part = slice(at, at + 40)
        z, size = X[part].double() @ w.T, X[part].double().abs() @ w.abs().T
        within(Y[part], z, half_step(t) * z.abs() * 1.01 + (K + 2) * STEP * size, "Y")
    del Y
    kept = qb.qb_checkpoint_act(X)
    dX, dW, db = qb.qb_linear_bwd(dY, kept, W)
    for at in places(max(N, K)):
        part = slice(at, at + 40)
        g, size = dY[part].double() @ w, dY[part].double().abs() @ w.abs()
        within(dX[part], g, half_step(t) * g.abs() * 1.01 + (N + 2) * STEP * size, "dX")
    # sums over all rows: of n numbers in binary32 in any order within n half steps of the sum of their magnitudes; X from 8 bits is rounded to `t`
    want, size, sums, sizes = 0.0, 0.0, 0.0, 0.0
    for at in range(0, T, 1 << 16):
        part = slice(at, at + (1 << 16))
        x = qb.qb_restore_act(kept[0][part], kept[1][part], t).double()
        d = dY[part].double()
        want, size, sums, sizes = want + d.T @ x, size + d.abs().T @ x.abs(), sums + d.sum(0), sizes + d.abs().sum(0)
    within(dW, want, half_step(t) * want.abs() * 1.01 + (T + 2) * STEP * size, "dW")
    within(db, sums, (T + 2) * STEP * sizes, "dbias")
