"""Layer norm, 16-bit linears and 8-bit activations on the host: workspace sizes, and every refusal comes before a launch (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_1909_05840_amd as qb

P, AT4, AT2, ODD = 0x1000, 0x1004, 0x1002, 0x1001  # addresses that are checked and never read
BF16, FP16, FP32 = 0, 1, 2
OK, NULL, SHAPE, VALUE, WORKSPACE = 0, 1, 3, 7, 5
f = ctypes.c_float
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return qb.load_library()


def test_checkpoints(lib):
    good = dict(X=P, row=100, type=BF16, T=5, W=100, codes=P, scales=P)
    for changed, status in ((dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(T=-1), SHAPE), (dict(T=2 ** 24 + 1), SHAPE), (dict(W=0), SHAPE),
                            (dict(W=32769), SHAPE), (dict(type=3), VALUE), (dict(type=-1), VALUE), (dict(X=ODD), VALUE), (dict(X=AT2, type=FP32), VALUE), (dict(scales=AT2), VALUE)):
        a = dict(good, **changed)
        assert lib.qb_checkpoint_act(a["X"], a["row"], a["type"], a["T"], a["W"], a["codes"], a["scales"], None) == status
        assert lib.qb_restore_act(a["codes"], a["scales"], a["T"], a["W"], a["type"], a["X"], None) == status
    for row in (-1, 2 ** 22 + 1):
        assert lib.qb_checkpoint_act(P, row, BF16, 5, 100, P, P, None) == VALUE
    assert lib.qb_checkpoint_act(None, 100, BF16, 0, 100, None, None, None) == OK
    assert lib.qb_restore_act(None, None, 0, 100, BF16, None, None) == OK


def test_layer_norm(lib):
    good = dict(X=P, row=100, type=FP32, T=5, W=100, weight=P, bias=P, eps=1e-5, Y=P, mean=P, rstd=P, codes=P, scales=P)
    for changed, status in ((dict(X=None), NULL), (dict(Y=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL),
                            (dict(T=-1), SHAPE), (dict(T=2 ** 24 + 1), SHAPE), (dict(W=0), SHAPE), (dict(W=32769), SHAPE), (dict(type=7), VALUE), (dict(eps=-1.0), VALUE),
                            (dict(eps=INF), VALUE), (dict(eps=NAN), VALUE), (dict(row=-1), VALUE), (dict(X=AT2), VALUE), (dict(Y=AT2), VALUE), (dict(weight=AT2), VALUE),
                            (dict(bias=ODD), VALUE), (dict(mean=AT2), VALUE), (dict(rstd=AT2), VALUE), (dict(scales=AT2), VALUE)):
        a = dict(good, **changed)
        assert lib.qb_layer_norm_fwd(a["X"], a["row"], a["type"], a["T"], a["W"], a["weight"], a["bias"], f(a["eps"]), a["Y"], a["mean"], a["rstd"], a["codes"], a["scales"], None) == status
    assert lib.qb_layer_norm_fwd(None, 100, BF16, 0, 100, None, None, f(1e-5), None, None, None, None, None, None) == OK


def norm(**changed):
    n = dict(dY=P, X=P, x_codes=None, x_scales=None, residual=None, dy_row=100, x_row=100, residual_row=0, weight=P, mean=P, rstd=P, type=BF16, T=50, W=100)
    n.update(changed)
    return ctypes.byref(qb.binding.NormGrads(**n))


def test_layer_norm_backward(lib):
    for changed, status in ((dict(dY=None), NULL), (dict(X=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL), (dict(x_codes=P, x_scales=P), NULL),
                            (dict(X=None, x_codes=P), NULL), (dict(x_scales=P), NULL), (dict(T=-1), SHAPE), (dict(W=0), SHAPE), (dict(W=40000), SHAPE), (dict(type=3), VALUE),
                            (dict(dy_row=-1), VALUE), (dict(x_row=2 ** 22 + 1), VALUE), (dict(residual_row=-4), VALUE), (dict(dY=ODD), VALUE), (dict(X=ODD), VALUE),
                            (dict(residual=ODD), VALUE), (dict(weight=AT2), VALUE), (dict(mean=AT2), VALUE)):
        assert lib.qb_layer_norm_bwd(norm(**changed), P, P, P, P, None) == status
    assert lib.qb_layer_norm_bwd(None, P, P, P, P, None) == NULL
    assert lib.qb_layer_norm_bwd(norm(), None, P, P, P, None) == NULL
    assert lib.qb_layer_norm_bwd(norm(), ODD, P, P, P, None) == VALUE
    assert lib.qb_layer_norm_bwd(norm(), P, AT2, P, P, None) == VALUE
    assert lib.qb_layer_norm_bwd(norm(), P, P, P, None, None) == WORKSPACE
    assert lib.qb_layer_norm_bwd(norm(), P, P, None, 0x1010, None) == WORKSPACE
    assert lib.qb_layer_norm_bwd_workspace_nbytes(-1, 8) == 0 and lib.qb_layer_norm_bwd_workspace_nbytes(8, 0) == 0
    assert lib.qb_layer_norm_bwd_workspace_nbytes(1, 8) >= 64


def linear(**changed):
    l = dict(type=BF16, act=0, T=390, N=768, K=768, X=P, x_row=768, W=P, bias=P, residual=P, residual_row=768, Y=P, pre=None, codes=P, scales=P)
    l.update(changed)
    return ctypes.byref(qb.binding.LinearLayer(**l))


LINEAR = [(dict(X=None), NULL), (dict(W=None), NULL), (dict(Y=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(T=-1), SHAPE), (dict(T=2 ** 24 + 1), SHAPE),
          (dict(N=0), SHAPE), (dict(N=2 ** 20 + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=100), SHAPE), (dict(K=32832), SHAPE), (dict(type=FP32), VALUE), (dict(type=-1), VALUE),
          (dict(act=4), VALUE), (dict(act=-1), VALUE), (dict(x_row=772), VALUE), (dict(x_row=-8), VALUE), (dict(x_row=2 ** 22 + 8), VALUE), (dict(residual_row=-1), VALUE),
          (dict(pre=P), VALUE), (dict(X=0x1008), VALUE), (dict(W=0x1008), VALUE), (dict(Y=ODD), VALUE), (dict(residual=ODD), VALUE), (dict(bias=AT2), VALUE),
          (dict(scales=AT2), VALUE), (dict(act=1, pre=ODD), VALUE)]


@pytest.mark.parametrize("changed, status", LINEAR)
def test_linear_refuses(lib, changed, status):
    assert lib.qb_linear_fwd(linear(**changed), P, None) == status


def test_linear_workspace(lib):
    assert lib.qb_linear_fwd(None, P, None) == NULL and lib.qb_linear_bwd(None, P, None) == NULL
    assert lib.qb_linear_fwd_workspace_nbytes(None) == 0 and lib.qb_linear_bwd_workspace_nbytes(None) == 0
    assert lib.qb_linear_fwd(linear(T=0, X=None, Y=None), None, None) == OK
    for T, N, K in ((390, 768, 768), (64, 1024, 4096), (16384, 4096, 1024), (1, 1, 64)):
        n = lib.qb_linear_fwd_workspace_nbytes(linear(T=T, N=N, K=K, x_row=K))
        assert n % 256 == 0 and n <= 64 * T * (N + 63)
        if n:
            assert lib.qb_linear_fwd(linear(T=T, N=N, K=K, x_row=K), None, None) == WORKSPACE
            assert lib.qb_linear_fwd(linear(T=T, N=N, K=K, x_row=K), 0x1010, None) == WORKSPACE
    assert lib.qb_linear_fwd_workspace_nbytes(linear(K=100)) == 0


def grads(**changed):
    g = dict(type=BF16, act=0, T=390, N=768, K=768, dY=P, dy_row=768, W=P, X=P, x_row=768, x_codes=None, x_scales=None, pre=None, pre_codes=None, pre_scales=None, dX=P, dW=P, dbias=P)
    g.update(changed)
    return ctypes.byref(qb.binding.LinearGrads(**g))


GRADS = [(dict(dY=None), NULL), (dict(W=None), NULL), (dict(X=None), NULL), (dict(X=None, x_codes=P), NULL), (dict(x_scales=P), NULL), (dict(act=1, pre_codes=P), NULL),
         (dict(T=-1), SHAPE), (dict(N=0), SHAPE), (dict(N=2 ** 20 + 1), SHAPE), (dict(K=96), SHAPE), (dict(type=FP32), VALUE), (dict(act=9), VALUE), (dict(x_row=4), VALUE),
         (dict(dy_row=-1), VALUE), (dict(act=1), VALUE), (dict(pre=P), VALUE), (dict(act=1, pre=P, pre_codes=P, pre_scales=P), VALUE), (dict(x_codes=P, x_scales=P), VALUE),
         (dict(dY=ODD), VALUE), (dict(W=0x1008), VALUE), (dict(X=0x1008), VALUE), (dict(dX=ODD), VALUE), (dict(dW=ODD), VALUE), (dict(dbias=AT2), VALUE), (dict(act=1, pre=ODD), VALUE)]


@pytest.mark.parametrize("changed, status", GRADS)
def test_linear_backward_refuses(lib, changed, status):
    assert lib.qb_linear_bwd(grads(**changed), P, None) == status


def test_linear_backward_workspace(lib):
    kept = dict(X=None, x_codes=P, x_scales=P)  # (X in 16 bits has to lie somewhere)
    assert lib.qb_linear_bwd_workspace_nbytes(grads(**kept)) >= 390 * 768 * 2
    assert lib.qb_linear_bwd(grads(**kept), None, None) == WORKSPACE and lib.qb_linear_bwd(grads(**kept), 0x1080, None) == WORKSPACE
    for T, N, K in ((1, 1, 64), (390, 768, 768), (16384, 4096, 1024), (16384, 2, 1024), (1 << 24, 1, 64)):
        for more in (dict(), dict(X=None, x_codes=P, x_scales=P), dict(dX=None), dict(dW=None, X=None), dict(dX=None, dW=None), dict(dy_row=N + 1)):
            n = lib.qb_linear_bwd_workspace_nbytes(grads(T=T, N=N, K=K, dy_row=more.pop("dy_row", N), x_row=K, **more))
            assert n % 256 == 0 and n <= 200 * (T + 256) * (N + 64) + 40 * 4 * (T + N + 256) * K


def test_binding_refuses_what_is_not_on_the_gpu():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    v = torch.zeros(4)
    with pytest.raises(TypeError):
        qb.qb_linear_fwd(x, w)
    with pytest.raises(TypeError):
        qb.qb_linear_bwd(x, x, w)
    with pytest.raises(TypeError):
        qb.qb_layer_norm_fwd(x)
    with pytest.raises(TypeError):
        qb.qb_layer_norm_bwd(x, x, None, v, v)
    with pytest.raises(TypeError):
        qb.qb_checkpoint_act(x)
    with pytest.raises(ValueError):
        qb.qb_linear_fwd(x, w, act="swish")
    with pytest.raises(ValueError):
        qb.qb_linear_bwd(x, x, w, act="swish")
