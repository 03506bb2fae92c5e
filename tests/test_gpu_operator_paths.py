"""Paths of the attention backward and of the vocabulary loss that small calls do not take."""
import math

import pytest
import torch

import test_gpu_attention
import test_gpu_vocab_loss
from test_gpu_attention import E32, TRAIN, keep64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


class Case(test_gpu_attention.Case):
    """The same calls with a bound that follows the kernels row by row.  delta = dO.O takes the rounded O, which is corrected but for products of two
    roundings at dim 64, and at dim 128 where the tile of 128 rows (tokens times the heads of a group) sees 1024 keys or less; else u of |dO|.|O| remains."""
    def corrected(self, nq, nk):
        """of a sequence's tokens and heads of a group: whether the row's tile is corrected"""
        row = torch.arange(nq * self.group, device=DEV)
        last = (row // 128 * 128 + 127) // self.group
        seen = (last.clamp(max=nq - 1) + 1 + nk - nq).clamp(0, nk) if self.causal else torch.full_like(row, nk)
        return ((seen <= 1024) | (self.dim == 64)).reshape(nq, self.group)

    def exact(self, backward=False):
        assert backward
        val = {n: torch.zeros(x.shape, dtype=torch.float64, device=DEV) for n, x in (("dQ", self.Q), ("dK", self.K), ("dV", self.V))}
        tol = {n: torch.zeros_like(x) for n, x in val.items()}
        seed = int(self.seed) if self.p else 0
        for b, (nq, nk) in enumerate(zip(self.q_lens, self.k_lens)):
            if nq == 0 or nk == 0:
                continue
            rq, rk = slice(self.cq[b], self.cq[b] + nq), slice(self.ck[b], self.ck[b] + nk)
            hidden = torch.zeros(nq, nk, dtype=torch.bool, device=DEV)
            if self.causal:
                hidden = torch.arange(nk, device=DEV)[None, :] > torch.arange(nq, device=DEV)[:, None] + nk - nq
            corrected = self.corrected(nq, nk)
            for h in range(self.heads):
                of = h // self.group
                q, k, v, d = self.Q[rq, h].double(), self.K[rk, of].double(), self.V[rk, of].double(), self.dO[rq, h].double()
                s = (q @ k.t() * self.scale).masked_fill(hidden, -math.inf)
                lse = torch.logsumexp(s, 1)
                P = torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[:, None])
                M = keep64(self.cq[b], nq, h, nk, self.p, seed)
                s_err = E32 / 4 * self.scale * (q.abs() @ k.abs().t())
                dP = (d @ v.t()) * M
                dS = P * (dP - (P * dP).sum(1, keepdim=True))
                d_abs = (d.abs() * ((P * M) @ v).abs()).sum(1, keepdim=True)
                off = torch.where(corrected[:, h % self.group], 8 * self.u ** 2, self.u)[:, None] * d_abs
                S_tol = 1.05 * self.u * dS.abs() + P * (E32 * ((d.abs() @ v.abs().t()) * M + d_abs) + off) + 2 * s_err * dS.abs()
                val["dQ"][rq, h] = dS @ k * self.scale
                tol["dQ"][rq, h] = S_tol @ k.abs() * self.scale
                val["dK"][rk, of] += dS.t() @ q * self.scale
                tol["dK"][rk, of] += S_tol.t() @ q.abs() * self.scale
                val["dV"][rk, of] += (P * M).t() @ d
                tol["dV"][rk, of] += (P * M * (1.05 * self.u + 2 * s_err)).t() @ d.abs()
        for n in val:
            tol[n] += self.u * val[n].abs() + 1e-6
        return val, tol


BACKWARD = dict(TRAIN)
for kind in ("bf16", "fp16"):
    BACKWARD["wide, more than 1024 keys, " + kind] = dict(type=kind, dim=128, heads=2, kv_heads=1, q_lens=[150, 70], k_lens=[1500, 1025])
    BACKWARD["wide, causal, rows on both sides of 1024 keys, " + kind] = dict(type=kind, dim=128, heads=3, kv_heads=1, q_lens=[1400, 30], causal=True, fused=True)
    BACKWARD["wide, causal, on both sides, dropout, " + kind] = dict(type=kind, dim=128, heads=2, kv_heads=2, q_lens=[1300], causal=True, p=0.2)
    BACKWARD["more keys than 2048, " + kind] = dict(type=kind, dim=64, heads=2, kv_heads=2, q_lens=[200], k_lens=[5000])
    BACKWARD["groups of eighty, " + kind] = dict(type=kind, dim=64, heads=80, kv_heads=1, q_lens=[33, 1, 40], causal=True)
    BACKWARD["groups of eighty, wide, dropout, " + kind] = dict(type=kind, dim=128, heads=160, kv_heads=2, q_lens=[20, 9], k_lens=[150, 9], p=0.1)
    BACKWARD["groups of 130, in parts, " + kind] = dict(type=kind, dim=64, heads=130, kv_heads=1, q_lens=[300], k_lens=[200], causal=True)


@pytest.mark.parametrize("name", BACKWARD)
def test_attention_backward(qb, name):
    say("attention backward:", name)
    c = Case(**BACKWARD[name])
    O, lse = c.forward(qb)
    grads = [torch.full(x.shape, float("nan"), dtype=c.dtype, device=DEV) for x in (c.Q, c.K, c.V)]
    c.backward(qb, O, lse, dQ=grads[0], dK=grads[1], dV=grads[2])
    val, tol = c.exact(backward=True)
    for n, x in zip(("dQ", "dK", "dV"), grads):
        test_gpu_attention.check(n, x, val[n], tol[n])
    assert all(torch.equal(x, y) for x, y in zip(grads, c.backward(qb, O, lse)))


# 20011 words are 79 tiles of 256 and 313 of 64: of 300 tokens 1565 tiles for 512 workgroups, of 1500 tokens 474 for 256
@pytest.mark.parametrize("K", [64, 128, 192, 256, 768])
@pytest.mark.parametrize("T,labelled,weights", [(300, 300, True), (512, 290, False), (513, 513, True), (1500, 1500, False), (3000, 1300, True)])
def test_a_workgroup_does_several_tiles_of_the_vocabulary(qb, T, labelled, weights, K):
    say("vocabulary loss:", labelled, "of", T, "tokens, 20011 words,", K, "units")
    c = test_gpu_vocab_loss.Case(T, 20011, K, labelled=labelled, weights=weights, std=0.5 * K ** -0.5)
    val, tol = c.exact()
    loss, lse = (torch.full(c.targets.shape, float("nan"), device=DEV) for _ in range(2))
    qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias, loss=loss, lse=lse)
    dX, dW, db = torch.full_like(c.X, float("nan")), torch.full_like(c.W, float("nan")), torch.full((20011,), float("nan"), device=DEV)
    qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias, dX=dX, dW=dW, dbias=db)
    for n, x in (("loss", loss), ("lse", lse), ("dX", dX), ("dW", dW), ("dbias", db)):
        test_gpu_vocab_loss.check(n, x, val[n], tol[n])
    again = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias) + qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)
    assert all(torch.equal(x, y) for x, y in zip(again, (loss, lse, dX, dW, db)))
