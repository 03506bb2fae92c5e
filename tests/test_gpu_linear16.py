"""Linears in 16 bits against 64 bits: every kernel's sizes and edges, epilogues, what is kept for the backward, gradients from 16 and from 8 bits."""
import pytest
import torch

import layer_reference as ref
from layer_reference import STEP, half_step, near

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
ACTS = [None, "gelu", "relu", "tanh"]


def weights(N, K, t):
    return ref.draw(N, K, seed=N + K, std=K ** -0.5, t=t), ref.draw(N, seed=7, std=0.5, t=torch.float32)


def rounded(t, value):
    """what the last rounding to `t` may be off, subnormal numbers included"""
    return half_step(t) * value.abs() * (1 + 2 * half_step(t)) + torch.finfo(t).tiny * torch.finfo(t).eps


def product(A, B):
    """A B^T in 64 bits, and what sums in binary32 in any order may be off"""
    a, b = A.double(), B.double()
    return a @ b.T, (A.shape[1] + 2) * STEP * (a.abs() @ b.abs().T)


def check_forward(qb, T, N, K, t, act=None, bias=True, residual=False, keep=None, wide=False):
    W, b = weights(N, K, t)
    X = ref.draw(T, K, seed=T, t=t)
    R = ref.draw(T, N, seed=T + 1, t=t) if residual else None
    z, off = product(X, W)
    if bias:
        z, off = z + b.double(), off + 2 * STEP * (z.abs() + b.double().abs())
    y, slope, own, _ = ref.act(act, z)
    off_y = 1.2 * off + own  # (no activation is steeper than 1.13)
    if residual:
        y, off_y = y + R.double(), off_y + 2 * STEP * (y.abs() + R.double().abs())
    x = X.cuda()
    if wide:
        x = torch.nn.functional.pad(x, (8, 24), value=float("nan"))[:, 8:8 + K]
    if residual and wide:
        R = torch.nn.functional.pad(R, (3, 2), value=float("nan"))[:, 3:3 + N]
    got = qb.qb_linear_fwd(x, W.cuda(), b.cuda() if bias else None, act=act, residual=None if R is None else R.cuda(), keep=keep)
    near(got if keep is None else got[0], y, rounded(t, y) + off_y, "Y")
    if keep == "codes":
        ref.check_kept(*got[1], *((z, off) if act else (y, off_y)))
    elif keep == "values":
        near(got[1], z, rounded(t, z) + off, "pre")


SIZES = [(1, 1, 64), (1, 4096, 1024), (2, 3, 128), (3, 65, 64), (7, 768, 768), (16, 130, 4096), (17, 1000, 192), (31, 64, 64), (32, 96, 32768), (33, 33, 128), (64, 1024, 4096),
         (129, 127, 64), (390, 768, 768), (390, 2304, 768), (257, 511, 1024), (1500, 1100, 128), (2000, 2100, 64), (4100, 3001, 64), (3, 70000, 64), (12001, 1024, 64), (40, 4100, 4096), (64, 4097, 2048), (8190, 1000, 128), (301, 2, 128), (5000, 3, 64), (70, 100, 32768)]


# tiles whose contraction is cut into parts: steps that do not come out even, a last group that is not whole, rows behind the last tile's
CUT = [(65, 1024, 4096), (390, 768, 3008), (200, 770, 4032), (70, 65, 32768), (65, 1, 576), (700, 200, 8192)]


@pytest.mark.parametrize("T,N,K", CUT)
@pytest.mark.parametrize("act,residual,keep,wide", [(None, False, None, False), ("gelu", True, "codes", True), (None, True, "codes", False), ("tanh", False, "values", False)])
def test_contractions_in_parts(qb, T, N, K, act, residual, keep, wide):
    check_forward(qb, T, N, K, torch.bfloat16 if N % 2 else torch.float16, act=act, residual=residual, keep=keep, wide=wide)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,N,K", SIZES)
def test_sizes(qb, t, T, N, K):
    check_forward(qb, T, N, K, t, act="gelu", residual=True, keep="codes")


@pytest.mark.parametrize("T,N", [(1, 200), (21, 77), (100, 72), (600, 1000), (1500, 1100), (4100, 3001)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [False, True])
def test_epilogues(qb, T, N, act, residual):
    for keep in (None, "codes", "values") if act else (None, "codes"):
        check_forward(qb, T, N, 128, torch.bfloat16, act=act, residual=residual, keep=keep, bias=keep != "codes")


@pytest.mark.parametrize("T,N,K", [(1, 64, 64), (20, 100, 4096), (300, 200, 512), (2100, 2048, 64)])
def test_rows_apart(qb, T, N, K):
    check_forward(qb, T, N, K, torch.float16, residual=True, wide=True)


def check_backward(qb, T, N, K, t, x="given", pre=None, act=None, wide=0, need=(True, True, True), std=1.0):
    W, _ = weights(N, K, t)
    dY = ref.draw(T, N, seed=3, t=t, std=std)
    X, kept, before = ref.draw(T, K, seed=5, t=t, std=1.5), None, None
    value = X.double()
    more = torch.zeros(())
    if x == "codes":
        kept = ref.keep(X)
        value = ref.restore(*kept)
        more = rounded(t, value)
    dX, off = product(dY, W.T.contiguous())
    if pre:
        z = X
        kept = ref.keep(z) if pre == "codes" else None
        before = ref.restore(*kept) if pre == "codes" else z.double()
        h, slope, own, own_slope = ref.act(act, before)
        off = off * slope.abs() + dX.abs() * (own_slope + 2 * STEP)
        dX = dX * slope
        if x == "again":
            value, more = h, rounded(t, h) * (1 + half_step(t)) + own
        else:
            value = X.double()
    dW, off_w = product(dY.T.contiguous(), value.T.contiguous())
    off_w = off_w + dY.double().abs().T @ (more + 0 * value)
    gpu = lambda v: v if v is None else tuple(i.cuda() for i in v)  # noqa: E731
    g = dY.cuda()
    if wide:
        g = torch.nn.functional.pad(g, (wide, 24 - wide), value=float("nan"))[:, wide:wide + N]
    xs = X.cuda()
    if wide:
        xs = torch.nn.functional.pad(xs, (8, 8), value=float("nan"))[:, 8:8 + K]
    arg = gpu(kept) if x == "codes" else None if x == "again" else xs
    p = None if not pre else gpu(kept) if pre == "codes" else X.cuda()
    got = qb.qb_linear_bwd(g, arg, W.cuda(), pre=p, act=act, need=need)
    want = (dX, dW, dY.double().sum(0))
    bound = (off + rounded(t, dX), off_w + rounded(t, dW), (T + 2) * STEP * dY.double().abs().sum(0))
    for k, name in enumerate(("dX", "dW", "dbias")):
        if need[k]:
            near(got[k], want[k], bound[k], name)
        else:
            assert got[k] is None


BACK = [(1, 1, 64), (1, 768, 128), (2, 3, 64), (5, 8, 192), (63, 64, 64), (64, 65, 64), (65, 72, 128), (127, 200, 4096), (130, 1000, 64), (390, 768, 768), (390, 2304, 256), (1000, 120, 1024),
        (1030, 2, 768), (129, 4100, 64), (2050, 1030, 1024), (2051, 2101, 704), (8200, 520, 576), (9, 2048, 2048), (33000, 16, 64)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,N,K", BACK)
def test_gradients(qb, t, T, N, K):
    check_backward(qb, T, N, K, t)


@pytest.mark.parametrize("T,N,K", [(1, 1, 64), (50, 66, 128), (700, 300, 320), (2050, 1030, 1024), (2051, 2101, 704)])
@pytest.mark.parametrize("x,pre,act", [("codes", None, None), ("again", "codes", "gelu"), ("again", "values", "gelu"), ("given", "codes", "tanh"), ("given", "values", "relu"),
                                       ("again", "codes", "relu"), ("again", "values", "tanh")])
def test_gradients_with_what_was_kept(qb, T, N, K, x, pre, act):
    for t in TYPES if T < 1000 else TYPES[:1]:
        check_backward(qb, T, N, K, t, x=x, pre=pre, act=act)


@pytest.mark.parametrize("wide", [8, 3])
@pytest.mark.parametrize("T,N,K", [(1, 8, 64), (70, 128, 128), (700, 333, 320), (2051, 2104, 704)])
def test_gradients_of_rows_apart(qb, T, N, K, wide):
    check_backward(qb, T, N, K, torch.bfloat16, wide=wide)


def test_the_same_row_for_every_token(qb):
    """a gradient that was broadcast, tokens that were: no stride between rows"""
    for T, N, K in ((40, 72, 64), (300, 200, 128), (2051, 2104, 704)):
        W, b = (v.cuda() for v in weights(N, K, torch.bfloat16))
        g, x = ref.draw(1, N, seed=1, t=torch.bfloat16).cuda().expand(T, N), ref.draw(1, K, seed=2, t=torch.bfloat16).cuda().expand(T, K)
        assert torch.equal(qb.qb_linear_fwd(x, W, b), qb.qb_linear_fwd(x.contiguous(), W, b))
        assert all(torch.equal(p, q) for p, q in zip(qb.qb_linear_bwd(g, x, W), qb.qb_linear_bwd(g.contiguous(), x.contiguous(), W)))


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True), (False, False, False)])
def test_only_some_gradients(qb, need):
    for T, N, K in ((40, 100, 64), (390, 768, 768), (2051, 2101, 704)):
        check_backward(qb, T, N, K, torch.bfloat16, need=need)
        check_backward(qb, T, N, K, torch.bfloat16, x="again", pre="codes", act="gelu", need=need)


def test_small_gradients_in_fp16(qb):
    check_backward(qb, 300, 200, 128, torch.float16, std=1e-6)  # (subnormal numbers)


def test_gradients_against_differences(qb):
    """of sum dY (act(pre) W^T + b) in 64 bits, in directions of pre, W and b"""
    T, N, K = 40, 70, 64
    W, b = weights(N, K, torch.float16)
    pre, dY = ref.draw(T, K, seed=1, t=torch.float16), ref.draw(T, N, seed=2, t=torch.float16)
    for act in ACTS[1:]:
        grads = [g.cpu().double() for g in qb.qb_linear_bwd(dY.cuda(), None, W.cuda(), pre=pre.cuda(), act=act)]

        def loss(p, w, c):
            return ((ref.act(act, p)[0] @ w.T + c) * dY.double()).sum()
        args = [pre.double(), W.double(), b.double()]
        for i in range(3):
            v = ref.draw(*args[i].shape, seed=30 + i)
            if act == "relu" and i == 0:
                v = torch.where(pre.double().abs() < 1e-3, 0.0, v)  # (a step across the corner)
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + 1e-4 * v, args[i] - 1e-4 * v
            slope = (loss(*up) - loss(*down)) / 2e-4
            # the quotient is off by about the step squared; every entry of a gradient by half a rounding step of fp16, those of act(pre) in dW by another
            assert abs(slope - (grads[i] * v).sum()) <= 1e-5 + 3 * half_step(torch.float16) * (grads[i] * v).abs().sum() + 1e-3 * (i == 1)


def test_nothing_behind_the_outputs_is_written(qb):
    for T, N, K in ((1, 3, 64), (33, 67, 64), (390, 769, 128), (4100, 3001, 64)):
        W, b = weights(N, K, torch.bfloat16)
        X = ref.draw(T, K, seed=1, t=torch.bfloat16)
        W, b, X = W.cuda(), b.cuda(), X.cuda()
        y = torch.full((T * N + 512,), 5.0, dtype=torch.bfloat16, device="cuda")
        pre = torch.full((T * N + 512,), 5.0, dtype=torch.bfloat16, device="cuda")
        codes = torch.full((T * N + 512,), 55, dtype=torch.int8, device="cuda")
        scales = torch.full((T * -(-N // 64) + 64,), 5.0, device="cuda")
        Y = y[:T * N].view(T, N)
        assert qb.qb_linear_fwd(X, W, b, act="gelu", keep="codes", Y=Y, kept=(codes[:T * N].view(T, N), scales[:-64].view(T, -1)))[0].data_ptr() == y.data_ptr()
        qb.qb_linear_fwd(X, W, b, act="gelu", keep="values", Y=Y, kept=pre[:T * N].view(T, N))
        assert (y[T * N:] == 5).all() and (pre[T * N:] == 5).all() and (codes[T * N:] == 55).all() and (scales[-64:] == 5).all()
        dx, dw, db = (torch.full((n + 512,), 5.0, dtype=d, device="cuda") for n, d in ((T * K, torch.bfloat16), (N * K, torch.bfloat16), (N, torch.float32)))
        qb.qb_linear_bwd(Y, X, W, dX=dx[:T * K].view(T, K), dW=dw[:N * K].view(N, K), dbias=db[:N])
        assert (dx[T * K:] == 5).all() and (dw[N * K:] == 5).all() and (db[N:] == 5).all()


@pytest.mark.parametrize("T,N,K", [(2, 1030, 4096), (24, 1024, 4096), (65, 1030, 4032), (390, 768, 768), (200, 130, 2048), (2051, 2101, 704)])
def test_workspaces_of_exactly_the_size(qb, T, N, K):
    import ctypes
    from paper_1909_05840_amd.binding import LinearGrads, LinearLayer
    lib = qb.load_library()
    W, b = weights(N, K, torch.bfloat16)
    X, dY = ref.draw(T, K, seed=1, t=torch.bfloat16).cuda(), ref.draw(T, N, seed=2, t=torch.bfloat16).cuda()
    W, b = W.cuda(), b.cuda()
    kept = tuple(v.cuda() for v in ref.keep(X.cpu()))

    def guarded(bytes):
        room = torch.full((bytes + 2048,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, whatever it is read as)
        start = 1024 + (-room.data_ptr()) % 256 if room.data_ptr() % 256 else 1024
        return room, room[start:start + bytes], start
    l = LinearLayer(type=0, act=0, T=T, N=N, K=K, X=X.data_ptr(), x_row=K, W=W.data_ptr(), bias=b.data_ptr())
    n = lib.qb_linear_fwd_workspace_nbytes(ctypes.byref(l))
    want = qb.qb_linear_fwd(X, W, b)
    if n:
        room, ws, start = guarded(n)
        assert torch.equal(qb.qb_linear_fwd(X, W, b, workspace=ws), want)
        assert (room[:start] == 0xFF).all() and (room[start + n:] == 0xFF).all()
    out = torch.empty(T * K + N * K, dtype=torch.bfloat16, device="cuda")
    g = LinearGrads(type=0, act=2, T=T, N=N, K=K, dY=dY.data_ptr(), dy_row=N, W=W.data_ptr(), pre_codes=kept[0].data_ptr(), pre_scales=kept[1].data_ptr(), dX=out.data_ptr(),
                    dW=out.data_ptr() + 2 * T * K, dbias=b.data_ptr())
    n = lib.qb_linear_bwd_workspace_nbytes(ctypes.byref(g))
    want = qb.qb_linear_bwd(dY, None, W, pre=kept, act="gelu")
    room, ws, start = guarded(n)
    got = qb.qb_linear_bwd(dY, None, W, pre=kept, act="gelu", workspace=ws)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (room[:start] == 0xFF).all() and (room[start + n:] == 0xFF).all()


def test_rows_stay_apart(qb):
    """infinities and NaN in one token reach that token's row only; in dY they reach dW and dbias too, as the formulas say"""
    for T in (3, 20, 300):
        W, b = weights(200, 128, torch.bfloat16)
        W, b = W.cuda(), b.cuda()
        X = ref.draw(T, 128, seed=1, t=torch.bfloat16).cuda()
        clean = qb.qb_linear_fwd(X, W, b, act="gelu", keep="codes")
        X[1, 5], X[2, 9] = float("nan"), float("inf")
        Y, (codes, scales) = qb.qb_linear_fwd(X, W, b, act="gelu", keep="codes")
        others = [i for i in range(T) if i not in (1, 2)]
        assert torch.equal(Y[others], clean[0][others]) and torch.equal(codes[others], clean[1][0][others])
        assert Y[1].isnan().all() and torch.equal(Y[2].float(), torch.where(W[:, 9] > 0, float("inf"), 0.0))  # (GELU's limits)
        assert qb.qb_restore_act(codes, scales)[1:3].isnan().all()


def test_no_rows(qb):
    W, b = weights(30, 64, torch.bfloat16)
    W, b = W.cuda(), b.cuda()
    X = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    Y, (codes, scales) = qb.qb_linear_fwd(X, W, b, act="gelu", keep="codes")
    assert Y.shape == (0, 30) and codes.shape == (0, 30) and scales.shape == (0, 1)
    dX, dW, db = qb.qb_linear_bwd(Y, X, W)
    assert dX.shape == (0, 64) and (dW == 0).all() and (db == 0).all()


def test_residual_in_place(qb):
    for T, N, K in ((4, 100, 64), (390, 768, 768), (2100, 2048, 64)):
        W, b = weights(N, K, torch.bfloat16)
        X, R = ref.draw(T, K, seed=1, t=torch.bfloat16).cuda(), ref.draw(T, N, seed=2, t=torch.bfloat16).cuda()
        want = qb.qb_linear_fwd(X, W.cuda(), b.cuda(), residual=R)
        assert torch.equal(qb.qb_linear_fwd(X, W.cuda(), b.cuda(), residual=R, Y=R), want)


@pytest.mark.parametrize("T,N,K", [(1, 4096, 1024), (2, 1024, 4096), (24, 1024, 4096), (390, 768, 768), (390, 768, 3008), (2051, 2101, 704)])
def test_graphs_and_streams(qb, T, N, K):
    W, b = (v.cuda() for v in weights(N, K, torch.bfloat16))
    X, dY = ref.draw(T, K, seed=1, t=torch.bfloat16).cuda(), ref.draw(T, N, seed=2, t=torch.bfloat16).cuda()
    kept = qb.qb_checkpoint_act(X)

    def step():
        return (*qb.qb_linear_fwd(X, W, b, act="gelu", keep="values"), *qb.qb_linear_bwd(dY, None, W, pre=kept, act="gelu"))
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(3):
        X.copy_(ref.draw(T, K, seed=10 + seed, t=torch.bfloat16))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    side = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    torch.cuda.synchronize()
    for s in side:
        with torch.cuda.stream(s):
            outs.append(step())
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(x, y) for x, y in zip(o, want))
