"""A small causal language model trained and served with the library's operators.

Every linear layer's master weights are quantized group by group at each step and its inputs to 8 bits
(straight-through backward, Sec. 3.1 of arXiv 1909.05840); attention runs over packed sequences of different lengths,
with dropout of its weights; dropout and the residual addition are one call; the loss goes from hidden states to
the vocabulary without the logits.  Afterwards the model continues prompts word by word over a cache of keys and values.

The text is synthetic: each sequence counts up by one, modulo `count`, from a random start.

    python examples/language_model.py [--steps 80]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_1909_05840_amd as qb  # noqa: E402

CLIP = qb.workloads.ACT_CLIP


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, bits, groups):
        packed, h, _, rs_w = qb.qb_quantize_groupwise(W, bits, groups)
        Xq, rs_x = qb.qb_quantize_act(X.contiguous(), CLIP)
        ctx.save_for_backward(Xq, packed, h)
        ctx.layer = bits, groups
        return qb.qb_qlinear_fwd(Xq, rs_x, CLIP, packed, h, rs_w, bits, groups, W.shape[0])

    @staticmethod
    def backward(ctx, dY):
        Xq, packed, h = ctx.saved_tensors
        dX, dW = qb.qb_qlinear_bwd_ste(dY.bfloat16().contiguous(), Xq, CLIP, packed, h, *ctx.layer)
        return dX.float(), dW, None, None


class Attention(torch.autograd.Function):
    """qkv [T, 3 * heads, dim] bf16 as the projection writes it; the gradient goes into one tensor of that shape."""
    @staticmethod
    def forward(ctx, qkv, cu, longest, p, seed):
        q, k, v = qkv.chunk(3, dim=1)
        O, lse = qb.qb_attention_fwd(q, k, v, cu, cu, longest, longest, causal=True, p=p, seed=seed)
        ctx.save_for_backward(qkv, cu, seed, O, lse)
        ctx.call = longest, p
        return O

    @staticmethod
    def backward(ctx, dO):
        qkv, cu, seed, O, lse = ctx.saved_tensors
        longest, p = ctx.call
        d = torch.empty_like(qkv)
        qb.qb_attention_bwd(dO.contiguous(), *qkv.chunk(3, dim=1), O, lse, cu, cu, longest, longest, causal=True, p=p, seed=seed,
                            **dict(zip(("dQ", "dK", "dV"), d.chunk(3, dim=1))))
        return d, None, None, None, None


class DropoutAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, residual, p, seed):
        ctx.save_for_backward(seed)
        ctx.p = p
        return qb.qb_dropout_fwd(X, p, seed, residual)

    @staticmethod
    def backward(ctx, dY):
        return qb.qb_dropout_bwd(dY.contiguous(), ctx.p, *ctx.saved_tensors), dY, None, None


class VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, bias, targets):
        loss, lse = qb.qb_vocab_loss_fwd(X, W, targets, bias)
        ctx.save_for_backward(X, W, bias, targets, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        X, W, bias, targets, lse = ctx.saved_tensors
        return *qb.qb_vocab_loss_bwd(dloss.contiguous(), X, W, targets, lse, bias), None


class Model(torch.nn.Module):
    def __init__(self, vocab, hidden=128, heads=2, layers=2, room=96, bits=8, groups=64):
        super().__init__()
        self.heads, self.layers, self.room, self.bits, self.groups = heads, layers, room, bits, groups
        self.words = torch.nn.Parameter(torch.randn(vocab, hidden) * 0.05)
        self.places = torch.nn.Parameter(torch.randn(room, hidden) * 0.05)
        self.bias = torch.nn.Parameter(torch.zeros(vocab))
        shapes = {"qkv": (3 * hidden, hidden), "out": (hidden, hidden), "up": (4 * hidden, hidden), "down": (hidden, 4 * hidden)}
        self.weights = torch.nn.ParameterDict({"%s%d" % (name, i): torch.nn.Parameter(torch.randn(shape) * shape[1] ** -0.5)
                                               for i in range(layers) for name, shape in shapes.items()})

    def norm(self, x):
        return F.layer_norm(x, x.shape[-1:])

    def hidden(self, words, places, attend, p=0.0, seeds=None):
        """attend(layer, qkv) -> what the attention gives; seeds: two a layer for the dropouts here."""
        lin = lambda name, x: Linear.apply(x, self.weights[name], self.bits, self.groups)  # noqa: E731
        add = (lambda x, y, s: DropoutAdd.apply(x, y, p, seeds[s:s + 1])) if p else (lambda x, y, s: x + y)
        x = self.norm(self.words[words] + self.places[places])
        for i in range(self.layers):
            qkv = lin("qkv%d" % i, x).bfloat16().view(len(words), 3 * self.heads, -1)
            a = lin("out%d" % i, attend(i, qkv).float().flatten(1))
            x = self.norm(add(a, x, 2 * i))
            x = self.norm(add(lin("down%d" % i, F.gelu(lin("up%d" % i, x))), x, 2 * i + 1))
        return x

    def loss(self, words, targets, cu, longest, p, seeds):
        """Mean loss of packed sequences; targets outside the vocabulary count nothing.  seeds: three a layer."""
        places = torch.cat([torch.arange(n, device=words.device) for n in cu.diff().tolist()])
        drop, weights = seeds[:2 * self.layers], seeds[2 * self.layers:]
        x = self.hidden(words, places, lambda i, qkv: Attention.apply(qkv, cu, longest, p, weights[i:i + 1]), p, drop)
        losses = VocabLoss.apply(x.bfloat16(), self.words.bfloat16(), self.bias, targets)
        return losses.sum() / (targets >= 0).sum()

    def cache(self, n_seqs):
        shape = self.layers, 2, n_seqs * self.room, self.heads, self.words.shape[1] // self.heads
        return torch.empty(shape, dtype=torch.bfloat16, device=self.words.device)

    @torch.no_grad()
    def extend(self, cache, lengths, words, cu, longest):
        """Appends new words (packed, `longest` at most of a sequence) to sequences of `lengths` words in the cache; returns the new lengths and the most likely
        next word of each sequence.  The same call takes whole prompts and single words."""
        n_seqs, dev = len(lengths), words.device
        new = cu.diff()
        seq = torch.repeat_interleave(torch.arange(n_seqs, device=dev), new.long())
        places = torch.arange(len(words), device=dev) - cu[seq] + lengths[seq]
        rows = seq * self.room + places
        lengths = lengths + new
        starts = torch.arange(n_seqs + 1, dtype=torch.int32, device=dev) * self.room

        def attend(i, qkv):
            q, k, v = qkv.chunk(3, dim=1)
            cache[i, 0, rows], cache[i, 1, rows] = k, v
            return qb.qb_attention_fwd(q, cache[i, 0], cache[i, 1], cu, starts, longest, self.room, causal=True, k_len=lengths)[0]

        x = self.hidden(words, places, attend)[cu[1:].long() - 1]
        return lengths, (x @ self.words.T + self.bias).argmax(1)


def texts(n, count, most, gen, dev):
    """n packed sequences of 2 .. most words that count up: words, targets, offsets."""
    lengths = torch.randint(2, most + 1, (n,), generator=gen)
    start = torch.randint(0, count, (n,), generator=gen)
    seqs = [(s + torch.arange(l)) % count for s, l in zip(start, lengths)]
    targets = [torch.cat([s[1:], torch.tensor([-1])]) for s in seqs]
    cu = F.pad(lengths.cumsum(0), (1, 0)).int()
    return torch.cat(seqs).to(dev), torch.cat(targets).to(dev), cu.to(dev)


def run(steps=80, n_seqs=24, vocab=499, count=61, most=64, p=0.1, new_words=8, verbose=True):
    """Trains and serves; returns (losses, share of right words among the continuations)."""
    dev = torch.device("cuda")
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(1)
    model = Model(vocab).to(dev)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    seeds = torch.arange(3 * model.layers, device=dev)
    losses = []
    for step in range(steps):
        words, targets, cu = texts(n_seqs, count, most, gen, dev)
        seeds += 1000  # other bits at each step
        loss = model.loss(words, targets, cu, most, p, seeds)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
        if verbose and (step % 10 == 0 or step == steps - 1):
            print("step %3d  loss %.3f" % (step, losses[-1]), flush=True)

    words, _, cu = texts(n_seqs, count, most, gen, dev)
    lengths, word = model.extend(cache := model.cache(n_seqs), torch.zeros(n_seqs, dtype=torch.int32, device=dev), words, cu, most)
    expected, one_each, right = words[cu[1:].long() - 1], torch.arange(n_seqs + 1, dtype=torch.int32, device=dev), 0
    for _ in range(new_words):
        expected = (expected + 1) % count
        right += (word == expected).sum().item()
        lengths, word = model.extend(cache, lengths, word, one_each, 1)
    share = right / (n_seqs * new_words)
    if verbose:
        print("%.1f%% of %d new words are right" % (100 * share, n_seqs * new_words))
    return losses, share


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=80)
    run(parser.parse_args().steps)
