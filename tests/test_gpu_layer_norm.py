"""Layer norm forward and backward against 64 bits: every width's kernel, types, rows apart, absent weights, 8-bit inputs and outputs."""
import pytest
import torch

import layer_reference as ref
from layer_reference import STEP, half_step, near

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1), (1, 768), (3, 7), (5, 64), (9, 65), (390, 768), (2050, 1000), (33, 1024), (7, 1025), (6, 2048), (5, 2049), (3, 4096), (4, 4097), (3, 8200), (2, 16385), (2, 32768), (4099, 24), (300, 8200), (131, 10000)]


def inputs(T, W, t):
    return ref.draw(T, W, seed=T + W, t=t, mean=0.3), ref.draw(W, seed=1, std=0.2, mean=1.0, t=torch.float32), ref.draw(W, seed=2, std=0.2, t=torch.float32)


def forward(X, w, b, eps):
    """in 64 bits: y, mean, rstd, h, and a bound of what binary32 makes y, and h, off (sums of W values over at most 64 additions a thread and sixteen more)"""
    x = X.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1 / (d.square().mean(1, keepdim=True) + eps).sqrt()
    h = d * rstd
    off = 100 * STEP * (rstd * (x.abs().mean(1, keepdim=True) + d.abs()))
    w, b = (1.0 if w is None else w.double()), (torch.zeros(()) if b is None else b.double())
    return h * w + b, mean[:, 0], rstd[:, 0], h, off, off * abs(w) + 4 * STEP * b.abs()


def backward(X, dY, w, h, off, rstd, past):
    """in 64 bits: dX, dw, db, and their bounds; `off`: of h"""
    dy = dY.double()
    w = torch.ones(X.shape[1], dtype=torch.float64) if w is None else w.double()
    g, r = dy * w, rstd[:, None]
    m0, m1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dX = r * (g - m0 - h * m1)
    a0, a1 = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    off_x = 100 * STEP * r * (g.abs() + a0 + h.abs() * a1) + r * (off * m1.abs() + h.abs() * (g.abs() * off).mean(1, keepdim=True))
    if past is not None:
        dX = dX + past.double()
        off_x = off_x + 4 * STEP * past.double().abs()
    off_w = len(X) * STEP * (dy * h).abs().sum(0) + (dy.abs() * off).sum(0) + 4 * STEP * (dy * h).abs().sum(0)
    return (dX, (dy * h).sum(0), dy.sum(0)), (off_x, off_w, (len(X) + 4) * STEP * dy.abs().sum(0))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,W", SHAPES)
def test_against_64_bits(qb, t, T, W):
    X, w, b = inputs(T, W, t)
    eps = 1e-5
    y, mean, rstd, h, off, off_y = forward(X, w, b, eps)
    Y, m, r, codes, scales = qb.qb_layer_norm_fwd(X.cuda(), w.cuda(), b.cuda(), eps, keep=True)
    near(Y, y, half_step(t) * y.abs() * (1 + 2 * half_step(t)) + off_y + torch.finfo(t).tiny * half_step(t) * 2, "Y")
    near(m, mean, 100 * STEP * X.double().abs().mean(1), "mean")
    near(r, rstd, 200 * STEP * rstd * (1 + rstd * X.double().abs().mean(1)), "rstd")
    ref.check_kept(codes, scales, y, off_y)
    dY, past = ref.draw(T, W, seed=3, std=0.5, t=t), ref.draw(T, W, seed=4, std=0.5, t=t)
    for p in (None, past):
        got = qb.qb_layer_norm_bwd(dY.cuda(), X.cuda(), w.cuda(), m, r, residual=None if p is None else p.cuda())
        want, bound = backward(X, dY, w, h, off + 200 * STEP * h.abs() * (1 + rstd * X.double().abs().mean(1))[:, None], rstd, p)
        near(got[0], want[0], half_step(t) * want[0].abs() * (1 + 2 * half_step(t)) + bound[0] + torch.finfo(t).tiny * half_step(t) * 2, "dX")
        near(got[1], want[1], bound[1], "dweight")
        near(got[2], want[2], bound[2], "dbias")


@pytest.mark.parametrize("t", TYPES)
def test_without_weight_and_bias(qb, t):
    X, w, b = inputs(19, 200, t)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, mean, rstd, h, off, off_y = forward(X, ww, bb, 1e-12)
        Y, m, r = qb.qb_layer_norm_fwd(X.cuda(), None if ww is None else ww.cuda(), None if bb is None else bb.cuda(), 1e-12)
        near(Y, y, half_step(t) * y.abs() * 1.01 + off_y + 1e-7, "Y")
        dY = ref.draw(19, 200, seed=3, t=t)
        got = qb.qb_layer_norm_bwd(dY.cuda(), X.cuda(), None if ww is None else ww.cuda(), m, r, sums=False)
        want, bound = backward(X, dY, ww, h, 3 * off, rstd, None)
        near(got[0], want[0], half_step(t) * want[0].abs() * 1.01 + bound[0] + 1e-7, "dX")
        assert got[1] is None and got[2] is None


def test_gradients_against_differences(qb):
    X, w, b = inputs(5, 40, torch.float32)
    dY = ref.draw(5, 40, seed=9, t=torch.float32)
    _, m, r = qb.qb_layer_norm_fwd(X.cuda(), w.cuda(), b.cuda(), 1e-5)
    dX, dw, db = (g.cpu().double() for g in qb.qb_layer_norm_bwd(dY.cuda(), X.cuda(), w.cuda(), m, r))

    def loss(x, w, b):
        return (torch.nn.functional.layer_norm(x, (40,), w, b, 1e-5) * dY.double()).sum()
    args = [X.double(), w.double(), b.double()]
    for i, grad in enumerate((dX, dw, db)):
        for k in range(3):
            v = ref.draw(*args[i].shape, seed=20 + k)
            step = 1e-4
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + step * v, args[i] - step * v
            slope = (loss(*up) - loss(*down)) / (2 * step)
            # the quotient's own error is of the order of step^2, the gradient's of a few hundred binary32 roundings
            assert abs(slope - (grad * v).sum()) <= 1e-6 * (1 + (grad * v).abs().sum())


def test_rows_apart(qb):
    wide, dwide, pwide = (ref.draw(50, 400, seed=s, t=torch.bfloat16).cuda() for s in (1, 2, 3))
    w = ref.draw(131, seed=4, t=torch.float32).cuda()
    part = (wide[:, 9:140], dwide[:, 100:231], pwide[:, 1:132])
    a = qb.qb_layer_norm_fwd(part[0], w)
    whole = [p.contiguous() for p in part]
    b = qb.qb_layer_norm_fwd(whole[0], w)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    ga = qb.qb_layer_norm_bwd(part[1], part[0], w, a[1], a[2], residual=part[2])
    gb = qb.qb_layer_norm_bwd(whole[1], whole[0], w, a[1], a[2], residual=whole[2])
    for x, y in zip(ga, gb):
        assert torch.equal(x, y)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,W", [(3, 65), (130, 768), (4, 2100)])
def test_backward_from_8_bits(qb, t, T, W):
    X, w, b = inputs(T, W, t)
    codes, scales = ref.keep(X)
    x = ref.restore(codes, scales)
    _, m, r = qb.qb_layer_norm_fwd(X.cuda(), w.cuda(), b.cuda())
    mean, rstd = m.cpu().double(), r.cpu().double()
    h = (x - mean[:, None]) * rstd[:, None]
    dY = ref.draw(T, W, seed=3, t=t)
    got = qb.qb_layer_norm_bwd(dY.cuda(), (codes.cuda(), scales.cuda()), w.cuda(), m, r)
    off = 8 * STEP * rstd[:, None] * (x.abs() + mean.abs()[:, None])
    want, bound = backward(X, dY, w, h, off, rstd, None)
    near(got[0], want[0], half_step(t) * want[0].abs() * 1.01 + bound[0] + 1e-7, "dX")
    near(got[1], want[1], bound[1], "dweight")
    near(got[2], want[2], bound[2], "dbias")


@pytest.mark.parametrize("T,W", [(100, 700), (50, 2000), (40, 9000), (12, 20000)])
def test_in_place(qb, T, W):
    X, w, b = inputs(T, W, torch.float16)
    X, w, b = X.cuda(), w.cuda(), b.cuda()
    Y, m, r = qb.qb_layer_norm_fwd(X, w, b)
    dY, past = ref.draw(T, W, seed=1, t=torch.float16).cuda(), ref.draw(T, W, seed=2, t=torch.float16).cuda()
    want = qb.qb_layer_norm_bwd(dY, X, w, m, r, residual=past)
    d = dY.clone()
    assert all(torch.equal(x, y) for x, y in zip(qb.qb_layer_norm_bwd(d, X, w, m, r, residual=past, dX=d), want))
    p = past.clone()
    assert torch.equal(qb.qb_layer_norm_bwd(dY, X, w, m, r, residual=p, dX=p)[0], want[0])
    x = X.clone()
    assert torch.equal(qb.qb_layer_norm_fwd(x, w, b, Y=x)[0], Y)


def test_far_from_zero(qb):
    # the squares are of x - mean: an offset of 2^12 standard deviations costs what binary32 loses in x itself
    X = ref.draw(20, 768, seed=6, mean=4096.0, t=torch.float32)
    y, _, rstd, _, off, off_y = forward(X, None, None, 1e-5)
    Y, _, r = qb.qb_layer_norm_fwd(X.cuda())
    near(Y, y, off_y + 1e-6, "Y")
    assert ((r.cpu().double() - rstd).abs() <= 1e-4 * rstd).all()


def test_no_rows_and_equal_rows(qb):
    w = torch.ones(100, device="cuda")
    Y, m, r = qb.qb_layer_norm_fwd(torch.empty(0, 100, device="cuda"), w)
    assert Y.shape == (0, 100) and m.shape == (0,)
    dX, dw, db = qb.qb_layer_norm_bwd(Y, Y, w, m, r)
    assert dX.shape == (0, 100) and (dw == 0).all() and (db == 0).all()
    X = torch.full((4, 100), 3.0, device="cuda")
    Y, m, r = qb.qb_layer_norm_fwd(X, w, eps=1e-12)
    assert (Y == 0).all() and (m == 3).all() and torch.allclose(r, torch.full_like(r, 1e6))


def test_many_rows_the_same_bits_and_graphs(qb):
    X = ref.draw(9001, 768, seed=1, t=torch.bfloat16).cuda()
    dY = ref.draw(9001, 768, seed=2, t=torch.bfloat16).cuda()
    w = torch.ones(768, device="cuda")
    _, m, r = qb.qb_layer_norm_fwd(X, w)
    first = qb.qb_layer_norm_bwd(dY, X, w, m, r)
    assert all(torch.equal(a, b) for a, b in zip(first, qb.qb_layer_norm_bwd(dY, X, w, m, r)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, m2, r2 = qb.qb_layer_norm_fwd(X, w)
        got = qb.qb_layer_norm_bwd(dY, X, w, m2, r2)
    for seed in range(3):
        X.copy_(ref.draw(9001, 768, seed=10 + seed, t=torch.bfloat16))
        graph.replay()
        want = qb.qb_layer_norm_fwd(X, w)
        grads = qb.qb_layer_norm_bwd(dY, X, w, want[1], want[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((Y, m2, r2) + tuple(got), tuple(want) + tuple(grads)))
