"""float16 has five bits of exponent: attention where weights and gradients lie below its normal numbers, or near its largest.

Results are rounded once, and what goes into their last product (P, dS) once before: two roundings of one size, sqrt(2) times the error of exact
arithmetic rounded once.  A tenth on top is for all the rest: exponentials, delta, sums in 32 bits."""
import math

import pytest
import torch

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOUND = 1.1 * math.sqrt(2.0)


def once(x, want):
    """how many times as far from `want` as `want` rounded to x's type"""
    return ((x.double() - want).norm() / (want.to(x.dtype).double() - want).norm()).item()


def check(what, x, want):
    off = once(x, want)
    print("  %s: %.2f times one rounding" % (what, off), flush=True)
    assert off < BOUND, what


CASES = {
    "many keys": dict(dim=64, heads=2, kv_heads=1, q_lens=[4096]),
    "short sequences": dict(dim=64, heads=4, kv_heads=4, q_lens=[384, 200, 65, 300], fused=True),
    "causal, wide": dict(dim=128, heads=3, kv_heads=1, q_lens=[1000, 130], causal=True),
    "dropout": dict(dim=64, heads=4, kv_heads=2, q_lens=[700, 384], p=0.1),
    "dropout, wide, causal": dict(dim=128, heads=2, kv_heads=2, q_lens=[900], p=0.5, causal=True),
}


@pytest.mark.parametrize("spread", [1e-4, 1e-3, 1e-2, 1.0, 100.0])
@pytest.mark.parametrize("name", CASES)
def test_gradients_of_any_size(qb, name, spread):
    print("float16 attention backward:", name, "dO of", spread, flush=True)
    c = Case("fp16", **CASES[name])
    c.dO = (c.dO.float() * spread).half()
    got = c.backward(qb, *c.forward(qb))
    val = c.exact(backward=True)[0]
    for n, x in zip(("dQ", "dK", "dV"), got):
        check(n, x, val[n])


@pytest.mark.parametrize("dim", [64, 128])
def test_sequences_heads_and_rows_of_different_sizes(qb, dim):
    """Sequences and key heads are apart; so are the rows of dQ, while dK and dV sum over a sequence's rows."""
    print("float16 attention backward: dO and V of many sizes", flush=True)
    c = Case("fp16", dim, 4, 2, [600, 500, 700])
    sizes = torch.tensor([1e-4, 1.0, 300.0], device=DEV).repeat_interleave(torch.tensor(c.q_lens, device=DEV))
    c.dO = (c.dO.float() * sizes[:, None, None]).half()
    c.V[:, 1] = (c.V[:, 1].float() * 2.0 ** -9).half()
    c.dO[::2, 3] = (c.dO[::2, 3].float() * 2.0 ** -8).half()
    got = dict(zip(("dQ", "dK", "dV"), c.backward(qb, *c.forward(qb))))
    val = c.exact(backward=True)[0]
    for b in range(3):
        rows = slice(c.cq[b], c.cq[b + 1])
        for n in got:
            for h in range(got[n].shape[1]):
                check("%s of sequence %d, head %d" % (n, b, h), got[n][rows, h], val[n][rows, h])
        check("small rows of dQ", got["dQ"][rows][::2, 3], val["dQ"][rows][::2, 3])


def test_weights_below_the_normal_numbers(qb):
    """40000 keys of about the same weight: P is 2^-15"""
    print("float16 attention backward: P of 2^-15", flush=True)
    c = Case("fp16", 64, 2, 1, [128], [40000], std=0.5)
    O, lse = c.forward(qb)
    val = c.exact(backward=True)[0]
    for n, x in zip(("O", "dQ", "dK", "dV"), (O,) + tuple(c.backward(qb, O, lse))):
        check(n, x, val[n])


def test_what_is_not_finite_stays_with_its_sequence(qb):
    print("float16 attention backward: infinity and NaN in one sequence's dO", flush=True)
    c = Case("fp16", 64, 2, 2, [300, 200])
    O, lse = c.forward(qb)
    want = [x[300:] for x in c.backward(qb, O, lse)]
    c.dO[3, 0, 5], c.dO[4, 1, 0] = float("inf"), float("nan")
    got = c.backward(qb, O, lse)
    assert all(torch.equal(x[300:], y) for x, y in zip(got, want))
    assert not torch.isfinite(got[1][:300]).any()
    c.dO[:300] = 0.0  # and nothing at all
    assert all((x[:300] == 0).all() and torch.equal(x[300:], y) for x, y in zip(c.backward(qb, O, lse), want))


@pytest.mark.parametrize("rows,heads,keys", [(1, 2, 500), (1, 2, 4096), (128, 32, 3000)])
@pytest.mark.parametrize("dim", [64, 128])
def test_weights_far_below_the_largest(qb, dim, rows, heads, keys):
    """The first key takes nearly all of the weight and has no value, as often in trained models; O is what the others give, each 2^-20 of it."""
    print("float16 attention: a first key of 2^20 times the weight", rows, heads, keys, dim, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(dim)
    Q = 1.0 + 0.01 * torch.randn(rows, heads, dim, generator=g, device=DEV)
    K, V = 0.3 * torch.randn(keys, heads, dim, generator=g, device=DEV), torch.randn(keys, heads, dim, generator=g, device=DEV)
    K[0], V[0] = 20 * math.log(2) / math.sqrt(dim), 0.0
    Q, K, V = Q.half(), K.half(), V.half()
    cu = [torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (rows, keys)]
    O, lse = qb.qb_attention_fwd(Q, K, V, *cu, rows, keys)
    q, k, v = (x.double().transpose(0, 1).contiguous() for x in (Q, K, V))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(dim)
    check("O", O.transpose(0, 1), torch.matmul(torch.softmax(s, 2), v))
    assert ((lse.t() - torch.logsumexp(s, 2)).abs() < 1e-5).all()
