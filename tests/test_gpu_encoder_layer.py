"""The operators together as an encoder layer uses them: linears with their epilogues, attention, layer norm, what the backward needs kept in 8 bits; against 64
bits, in graphs, and the same bits on another stream."""
import math

import pytest
import torch

from layer_reference import draw, half_step

pytestmark = pytest.mark.gpu
LENGTHS, HIDDEN, HEADS, INNER = [50, 100, 1, 29], 128, 2, 512
T = sum(LENGTHS)
SHAPES = {"qkv": (3 * HIDDEN, HIDDEN), "out": (HIDDEN, HIDDEN), "up": (INNER, HIDDEN), "down": (HIDDEN, INNER)}


def state(t, seed=0):
    s = {n: draw(*shape, seed=seed + i, std=shape[1] ** -0.5, t=t) for i, (n, shape) in enumerate(SHAPES.items())}
    s.update({"b_" + n: draw(shape[0], seed=seed + 10 + i, std=0.1, t=torch.float32) for i, (n, shape) in enumerate(SHAPES.items())})
    for i in (1, 2):
        s["w%d" % i], s["b%d" % i] = draw(HIDDEN, seed=seed + 20 + i, std=0.1, mean=1.0, t=torch.float32), draw(HIDDEN, seed=seed + 30 + i, std=0.1, t=torch.float32)
    s["x"], s["d"] = draw(T, HIDDEN, seed=seed + 40, t=t), draw(T, HIDDEN, seed=seed + 41, t=t)
    return s


def layer(qb, s, cu, keep=True):
    """forward and backward: out, then the gradients of x, the weights, the biases and the norms' parameters"""
    longest = max(LENGTHS)
    heads = lambda v: v.view(T, -1, HIDDEN // HEADS)  # noqa: E731
    qkv = heads(qb.qb_linear_fwd(s["x"], s["qkv"], s["b_qkv"]))
    q, k, v = qkv.chunk(3, dim=1)
    O, lse = qb.qb_attention_fwd(q, k, v, cu, cu, longest, longest)
    a = qb.qb_linear_fwd(O.view(T, HIDDEN), s["out"], s["b_out"], residual=s["x"])
    x1, m1, r1, *kept1 = qb.qb_layer_norm_fwd(a, s["w1"], s["b1"], keep=keep)
    h, kept_z = qb.qb_linear_fwd(x1, s["up"], s["b_up"], act="gelu", keep="codes" if keep else "values")
    y = qb.qb_linear_fwd(h, s["down"], s["b_down"], residual=x1)
    out, m2, r2 = qb.qb_layer_norm_fwd(y, s["w2"], s["b2"])

    dy, dw2, db2 = qb.qb_layer_norm_bwd(s["d"], y, s["w2"], m2, r2)
    dz, d_down, db_down = qb.qb_linear_bwd(dy, None, s["down"], pre=kept_z, act="gelu")
    dx1, d_up, db_up = qb.qb_linear_bwd(dz, tuple(kept1) if keep else x1, s["up"])
    da, dw1, db1 = qb.qb_layer_norm_bwd(dx1 + dy, a, s["w1"], m1, r1)
    dO, d_out, db_out = qb.qb_linear_bwd(da, O.view(T, HIDDEN), s["out"])
    d = torch.empty_like(qkv)
    qb.qb_attention_bwd(heads(dO), q, k, v, O, lse, cu, cu, longest, longest, **dict(zip(("dQ", "dK", "dV"), d.chunk(3, dim=1))))
    dx, d_qkv, db_qkv = qb.qb_linear_bwd(d.view(T, -1), s["x"], s["qkv"])
    return out, dx + da, d_qkv, d_out, d_up, d_down, db_qkv, db_out, db_up, db_down, dw1, db1, dw2, db2


def reference(s):
    p = {n: v.double().requires_grad_(n != "d") for n, v in s.items()}
    qkv = (p["x"] @ p["qkv"].T + p["b_qkv"]).view(T, 3 * HEADS, -1)
    q, k, v = qkv.chunk(3, dim=1)
    rows, at = [], 0
    for n in LENGTHS:
        part = slice(at, at + n)
        P = torch.softmax(torch.einsum("qhd,khd->hqk", q[part], k[part]) / math.sqrt(HIDDEN // HEADS), 2)
        rows.append(torch.einsum("hqk,khd->qhd", P, v[part]))
        at += n
    norm = torch.nn.functional.layer_norm
    x1 = norm(torch.cat(rows).reshape(T, HIDDEN) @ p["out"].T + p["b_out"] + p["x"], (HIDDEN,), p["w1"], p["b1"])
    y = torch.nn.functional.gelu(x1 @ p["up"].T + p["b_up"]) @ p["down"].T + p["b_down"] + x1
    out = norm(y, (HIDDEN,), p["w2"], p["b2"])
    names = ["x", "qkv", "out", "up", "down", "b_qkv", "b_out", "b_up", "b_down", "w1", "b1", "w2", "b2"]
    return [out.detach()] + list(torch.autograd.grad((out * p["d"]).sum(), [p[n] for n in names]))


def on_gpu(s):
    return {n: v.cuda() for n, v in s.items()}


def offsets():
    at = [0]
    for n in LENGTHS:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("keep", [True, False])
def test_against_64_bits(qb, t, keep):
    s = state(t)
    got, want = layer(qb, on_gpu(s), offsets(), keep), reference(s)
    # Norms of the differences.  Forward eight results are rounded on the way out (qkv, attention's weights and rows, a, x1, h, y, out), half a step each, and nothing on the way
    # amplifies them by more than two (a norm's division by a deviation of about one, GELU's slope of at most 1.13).  Backward sixteen at most are, and two of the
    # tensors that gradients are formed with are off by half a code: the largest of 64 values, below four deviations, over 254.
    for i, (g, w) in enumerate(zip(got, want)):
        bound = (2 * 8 if i == 0 else 2 * 16) * half_step(t) + (2 * 4 / 254 if keep and i > 0 else 0)
        off = (g.cpu().double() - w).norm() / w.norm()
        assert off <= bound, (i, float(off), bound)


def test_in_a_graph_and_on_another_stream(qb):
    s, cu = on_gpu(state(torch.bfloat16)), offsets()
    layer(qb, s, cu)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(qb, s, cu)
    for seed in (100, 200, 300):
        for n, v in state(torch.bfloat16, seed).items():
            s[n].copy_(v)
        graph.replay()
        want = layer(qb, s, cu)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = layer(qb, s, cu)
        again = layer(qb, s, cu)
    here = layer(qb, s, cu)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d) for a, b, c, d in zip(want, other, again, here))
