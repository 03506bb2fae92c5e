"""The operators round the quantized linears of an encoder or a small language model, as timed cases and a generator of
more of them.

  attention  softmax attention of packed sequences with grouped heads: an encoder's batch without padding, a causal prompt, a
             training step with dropout of the attention weights, and new tokens over a cache of earlier ones
  loss       softmax cross entropy behind the projection to the vocabulary, with the gradients of hidden states,
             embedding matrix and output bias; tokens whose target is no word (masked language modelling) have no loss
  dropout    dropout from a counter-based generator with the residual added, and its backward

Where `own` is false, `run` computes them from elementary tensor operations in 32 bits; where it is true, through the
public calls of `paper_1909_05840_amd`.

The random bits of dropout are Threefry-2x32 with 13 rounds (Salmon, Moraes, Dror, Shaw, SC 2011), key: the 64-bit seed.  One
counter gives four 16-bit draws (word 0 low and high half, then word 1); a value is dropped where its draw is below
round(p * 65536), and kept values are divided by the exact share that is kept.  Value i of a flat tensor takes draw i % 4 of
counter i // 4.  The weight of row q of the packed queries, head h, key k of its sequence takes draw k % 4 of the counter
(q, 2^31 + h * 2^22 + k // 4).
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
VOCAB = 30522


def listed():
    return [
        # the next token of four short requests, every head with keys of its own: launches and host work count
        {"name": "cache_4x1_bf16", "op": "cache", "type": "bf16", "seqs": 4, "new": 1, "cap": 390, "heads": 12, "kv_heads": 12, "dim": 64},
        # serving a batch of long conversations, grouped heads
        {"name": "cache_16x1_long_bf16", "op": "cache", "type": "bf16", "seqs": 16, "new": 1, "cap": 16384, "heads": 32, "kv_heads": 8, "dim": 128},
        # an encoder's batch of 32 requests of up to 512 tokens, without padding
        {"name": "encode_32x512_bf16", "op": "self", "train": False, "type": "bf16", "seqs": 32, "most": 512, "heads": 12, "kv_heads": 12, "dim": 64, "causal": False, "drop": 0.0},
        # causal prompts of odd lengths, grouped heads
        {"name": "prompt_3x3999_fp16", "op": "self", "train": False, "type": "fp16", "seqs": 3, "most": 3999, "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "drop": 0.0},
        # a fine-tuning step: 32 sequences of up to 384 tokens, attention weights dropped as BERT does
        {"name": "train_32x384_drop_bf16", "op": "self", "train": True, "type": "bf16", "seqs": 32, "most": 384, "heads": 12, "kv_heads": 12, "dim": 64, "causal": False, "drop": 0.1},
        # a training step of one long causal document
        {"name": "train_1x8192_bf16", "op": "self", "train": True, "type": "bf16", "seqs": 1, "most": 8192, "heads": 16, "kv_heads": 4, "dim": 64, "causal": True, "drop": 0.0},
        # masked language modelling on one short batch: 58 of 390 tokens have a target
        {"name": "loss_390tok_58", "op": "loss", "train": True, "tokens": 390, "labelled": 58, "hidden": 768, "vocab": VOCAB},
        # next-token training: every token of 16 x 512 has a target
        {"name": "loss_8192tok_all", "op": "loss", "train": True, "tokens": 8192, "labelled": 8192, "hidden": 1024, "vocab": VOCAB},
        # perplexity of a text, forward only
        {"name": "loss_eval_16384tok", "op": "loss", "train": False, "tokens": 16384, "labelled": 16000, "hidden": 768, "vocab": VOCAB},
        # masked language modelling, 32 x 512 tokens
        {"name": "loss_16384tok_2458", "op": "loss", "train": True, "tokens": 16384, "labelled": 2458, "hidden": 768, "vocab": VOCAB},
        # hidden dropout with the residual, one short sequence; 32-bit activations as the quantized linears give them
        {"name": "dropout_390x768_fp32", "op": "dropout", "type": "fp32", "tokens": 390, "hidden": 768, "drop": 0.1},
        # the same for a large batch in 16 bits
        {"name": "dropout_32768x1024_bf16", "op": "dropout", "type": "bf16", "tokens": 32768, "hidden": 1024, "drop": 0.1},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["cache", "cache", "self", "self", "self", "loss", "loss", "dropout"])
    if op == "dropout":
        return {"op": op, "type": rng.choice(["fp32", "bf16", "fp16"]), "tokens": _log_int(rng, 1, 32768), "hidden": rng.randint(1, 1024), "drop": rng.choice([0.05, 0.1, 0.5])}
    if op == "loss":
        tokens = _log_int(rng, 1, 8192)
        return {"op": op, "train": rng.random() < 0.7, "tokens": tokens, "labelled": max(1, tokens if rng.random() < 0.4 else int(tokens * rng.uniform(0.05, 1.0))),
                "hidden": 64 * rng.randint(2, 16), "vocab": _log_int(rng, 1000, VOCAB)}
    kv = rng.choice([1, 2, 4, 8, 12])
    c = {"op": op, "type": rng.choice(["bf16", "bf16", "fp16"]), "heads": kv * rng.choice([1, 1, 2, 3, 4] if kv < 12 else [1]), "kv_heads": kv, "dim": rng.choice([64, 64, 128])}
    if op == "cache":
        cap = _log_int(rng, 1, 16384)
        return {**c, "seqs": _log_int(rng, 1, min(16, 16 * 16384 * 8 * 128 // (cap * kv * c["dim"]))), "new": rng.choice([1, 1, 1, 2, 5]), "cap": cap}
    train = rng.random() < 0.5
    most = _log_int(rng, 2 if train else 1, 8192)  # (the weight of a lone token is 1: it has no gradient for queries and keys)
    # (the plain form works on padded squares: they bound the number of sequences)
    seqs = _log_int(rng, 1, max(1, min(64, int(16 * 8192 ** 2 / 4 / (c["heads"] * most ** 2)))))
    if c["heads"] * most ** 2 * c["dim"] > 16 * 8192 ** 2 * 64:
        most = int(math.sqrt(16 * 8192 ** 2 * 64 / (c["heads"] * c["dim"])))
    return {**c, "train": train, "seqs": seqs, "most": most, "causal": rng.random() < 0.5, "drop": 0.1 if train and most <= 4096 and rng.random() < 0.5 else 0.0}


def _lengths(n, most):
    """ragged: the first as long as allowed, the others spread over 1 .. most, the last of a larger batch empty"""
    got = [most] + [1 + int((most - 1) * (i * 0.6180339887498949 % 1.0)) for i in range(1, n)]
    if n > 3:
        got[-1] = 0
    return got


class _Draw:
    """tensors on the GPU from one seeded generator"""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, type=torch.float32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std).to(type)

    def seed64(self):
        return torch.randint(-(1 << 62), 1 << 62, (1,), generator=self.g, device="cuda", dtype=torch.int64)


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    rnd = _Draw(seed)
    s = dict(case)
    if case["op"] == "dropout":
        t = TYPES[case["type"]]
        shape = (case["tokens"], case["hidden"])
        s["X"], s["residual"] = rnd.normal(*shape, type=t), rnd.normal(*shape, type=t)
        s["dY"] = rnd.normal(*shape, std=1e-2, type=t)
        s["seed"] = rnd.seed64()
        return s
    if case["op"] == "loss":
        tokens, hidden, vocab = case["tokens"], case["hidden"], case["vocab"]
        s["X"] = rnd.normal(tokens, hidden, type=torch.bfloat16)  # behind a layer norm
        s["W"] = rnd.normal(vocab, hidden, std=0.04, type=torch.bfloat16)
        s["bias"] = rnd.normal(vocab, std=0.1)
        at = torch.randperm(tokens, generator=rnd.g, device="cuda")[:case["labelled"]]
        s["targets"] = torch.full((tokens,), -100, dtype=torch.int64, device="cuda")
        s["targets"][at] = torch.randint(0, vocab, (case["labelled"],), generator=rnd.g, device="cuda")
        s["dloss"] = torch.full((tokens,), 1.0 / case["labelled"], device="cuda")  # the mean over the tokens that have a target
        return s
    t, heads, kv, dim = TYPES[case["type"]], case["heads"], case["kv_heads"], case["dim"]
    s["scale"] = 1.0 / math.sqrt(dim)
    if case["op"] == "cache":
        lens = [max(case["new"], n) for n in _lengths(case["seqs"], case["cap"])]
        s["Q"] = rnd.normal(case["seqs"] * case["new"], heads, dim, std=1.4, type=t)
        s["K"], s["V"] = (rnd.normal(case["seqs"] * max(lens), kv, dim, std=w, type=t) for w in (1.4, 1.0))
        s["cu_q"], s["cu_k"] = _offsets([case["new"]] * case["seqs"]), _offsets([max(lens)] * case["seqs"])
        s["k_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["max_q"], s["max_k"], s["causal"], s["drop"], s["train"], s["seed"] = case["new"], max(lens), True, 0.0, False, None
        return s
    lens = _lengths(case["seqs"], case["most"])
    # queries, keys and values lie next to each other, as one projection writes them
    qkv = rnd.normal(sum(lens), heads + 2 * kv, dim, type=t)
    qkv[:, :heads + kv] *= 1.4
    s["Q"], s["K"], s["V"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    s["cu_q"] = s["cu_k"] = _offsets(lens)
    s["k_len"], s["max_q"], s["max_k"] = None, case["most"], case["most"]
    s["seed"] = rnd.seed64() if case["drop"] else None
    if case["train"]:
        s["dO"] = rnd.normal(sum(lens), heads, dim, std=1e-2, type=t)
    return s


# ---- the plain form: 32 bits, rounded once at the end ---------------------------------------------------------------

def _low(x):  # the low 32 bits as int32
    return ((x & 0xFFFFFFFF) ^ 0x80000000) - 0x80000000


def _draws(c0, c1, seed):
    """four 16-bit draws for each counter (c0, c1: int32 tensors that broadcast), in a last dimension"""
    k0, k1 = _low(seed).to(torch.int32), _low(seed >> 32).to(torch.int32)
    key = (k0, k1, k0 ^ k1 ^ 0x1BD11BDA)
    x0, x1 = torch.broadcast_tensors(c0 + key[0], c1 + key[1])
    for r in range(13):
        x0 = x0 + x1
        n = (13, 15, 26, 6, 17, 29, 16, 24)[r % 8]
        x1 = ((x1 << n) | ((x1 >> (32 - n)) & ((1 << n) - 1))) ^ x0
        if r % 4 == 3:
            x0 = x0 + key[(r // 4 + 1) % 3]
            x1 = x1 + (key[(r // 4 + 2) % 3] + (r // 4 + 1))
    return torch.stack((x0 & 0xFFFF, (x0 >> 16) & 0xFFFF, x1 & 0xFFFF, (x1 >> 16) & 0xFFFF), -1)


def _kept(draws, p):
    """one over the share that is kept where a value is kept, else zero"""
    threshold = min(65535, int(round(p * 65536)))
    return (draws >= threshold).float() * (65536.0 / (65536 - threshold))


def _plain_dropout(s):
    n = s["X"].numel()
    i = torch.arange((n + 3) // 4, device="cuda")
    scale = _kept(_draws(_low(i).to(torch.int32), (i >> 32).to(torch.int32), s["seed"]), s["drop"]).reshape(-1)[:n].reshape(s["X"].shape)
    return (s["X"].float() * scale + s["residual"].float()).to(s["X"].dtype), (s["dY"].float() * scale).to(s["dY"].dtype)


def _plain_loss(s):
    X, W = s["X"].float(), s["W"].float()
    has = s["targets"] >= 0
    at = s["targets"].clamp(min=0).unsqueeze(1)
    logits = X @ W.t() + s["bias"]
    top = logits.amax(1, keepdim=True)
    lse = top + (logits - top).exp().sum(1, keepdim=True).log()
    loss = torch.where(has, (lse - logits.gather(1, at)).squeeze(1), 0.0)
    kept = torch.where(has, lse.squeeze(1), 0.0)
    if not s["train"]:
        return loss, kept
    d = (logits - lse).exp()
    d.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    d *= torch.where(has, s["dloss"], 0.0).unsqueeze(1)
    return loss, kept, (d @ W).to(torch.bfloat16), (d.t() @ X).to(torch.bfloat16), d.sum(0)


def _plain_attention(s):
    Q, K, V, causal = s["Q"], s["K"], s["V"], s["causal"]
    heads, kv, dim = s["heads"], s["kv_heads"], s["dim"]
    seqs, mq, mk, g = s["seqs"], s["max_q"], s["max_k"], heads // kv
    q_at, k_at = s["cu_q"].long(), s["cu_k"].long()
    q_len = q_at[1:] - q_at[:-1]
    k_len = k_at[1:] - k_at[:-1] if s["k_len"] is None else s["k_len"].long()
    i, j = torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    has_q, has_k = i < q_len[:, None], j < k_len[:, None]  # [seqs, mq], [seqs, mk]
    row_q = torch.where(has_q, q_at[:-1, None] + i, 0)
    row_k = torch.where(has_k, k_at[:-1, None] + j, 0)
    # padded to [seqs, kv, g * mq, dim] and [seqs, kv, mk, dim]; head h of the queries reads head h // g of the keys
    pad_q = lambda x: (x.float()[row_q] * has_q[..., None, None]).reshape(seqs, mq, kv, g, dim).permute(0, 2, 3, 1, 4).reshape(seqs, kv, g * mq, dim)  # noqa: E731
    pad_k = lambda x: (x.float()[row_k] * has_k[..., None, None]).permute(0, 2, 1, 3).contiguous()  # noqa: E731
    unpad_q = lambda x: x.reshape(seqs, kv, g, mq, dim).permute(0, 3, 1, 2, 4).reshape(seqs, mq, heads, dim)[has_q].to(Q.dtype)  # noqa: E731
    unpad_k = lambda x: x.permute(0, 2, 1, 3)[has_k].to(K.dtype)  # noqa: E731
    sees = has_q[:, :, None] & has_k[:, None, :]
    if causal:  # the last query of a sequence sees all of its keys
        sees = sees & (j[None, None, :] <= i[None, :, None] + (k_len - q_len)[:, None, None])
    sees = sees[:, None, None].expand(seqs, 1, g, mq, mk).reshape(seqs, 1, g * mq, mk)
    q, k, v = pad_q(Q), pad_k(K), pad_k(V)
    logits = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~sees, -math.inf)
    top = logits.amax(3, keepdim=True).clamp(min=-3e38)
    P = logits.sub_(top).exp_()
    total = P.sum(3, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    P /= torch.where(total > 0, total, 1.0)
    if s["drop"]:
        h = torch.arange(heads, device="cuda").reshape(1, kv, g, 1, 1)
        c1 = _low((1 << 31) + h * (1 << 22) + torch.arange((mk + 3) // 4, device="cuda")).to(torch.int32)
        keep = _kept(_draws(row_q.to(torch.int32)[:, None, None, :, None], c1, s["seed"]).reshape(seqs, kv, g, mq, -1)[..., :mk], s["drop"]).reshape(P.shape)
        dropped = P * keep
    else:
        keep, dropped = 1.0, P
    out = torch.matmul(dropped, v)
    rows_lse = lse.reshape(seqs, kv, g, mq).permute(0, 3, 1, 2).reshape(seqs, mq, heads)[has_q]
    if not s["train"]:
        return unpad_q(out), rows_lse
    do = pad_q(s["dO"])
    dv = torch.matmul(dropped.transpose(2, 3), do)
    dP = torch.matmul(do, v.transpose(2, 3)) * keep
    dS = P * (dP - (P * dP).sum(3, keepdim=True)) * s["scale"]
    return unpad_q(out), rows_lse, unpad_q(torch.matmul(dS, k)), unpad_k(torch.matmul(dS.transpose(2, 3), q)), unpad_k(dv)


def run(s):
    op = s["op"]
    if not own:
        return _plain_dropout(s) if op == "dropout" else _plain_loss(s) if op == "loss" else _plain_attention(s)
    import paper_1909_05840_amd as qb
    if op == "dropout":
        return qb.qb_dropout_fwd(s["X"], s["drop"], s["seed"], residual=s["residual"]), qb.qb_dropout_bwd(s["dY"], s["drop"], s["seed"])
    if op == "loss":
        loss, lse = qb.qb_vocab_loss_fwd(s["X"], s["W"], s["targets"], bias=s["bias"])
        if not s["train"]:
            return loss, lse
        return (loss, lse) + tuple(qb.qb_vocab_loss_bwd(s["dloss"], s["X"], s["W"], s["targets"], lse, bias=s["bias"]))
    O, lse = qb.qb_attention_fwd(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"], causal=s["causal"], scale=s["scale"], k_len=s["k_len"], p=s["drop"], seed=s["seed"])
    if not s["train"]:
        return O, lse
    return (O, lse) + tuple(qb.qb_attention_bwd(s["dO"], s["Q"], s["K"], s["V"], O, lse, s["cu_q"], s["cu_k"], s["max_q"], s["max_k"], causal=s["causal"], scale=s["scale"], p=s["drop"], seed=s["seed"]))


def work(case):
    if case["op"] == "dropout":  # X, residual -> Y; dY -> dX
        return {"bytes": 5 * case["tokens"] * case["hidden"] * TYPES[case["type"]].itemsize, "flops": 0}
    if case["op"] == "loss":
        n, hidden, vocab = case["labelled"], case["hidden"], case["vocab"]
        weights, rows = 2 * vocab * hidden + 4 * vocab, 2 * n * hidden + 16 * case["tokens"]
        if not case["train"]:
            return {"bytes": weights + rows, "flops": 2 * n * hidden * vocab}
        return {"bytes": 2 * weights + 2 * rows + 2 * case["tokens"] * hidden, "flops": 6 * n * hidden * vocab}
    heads, kv, dim, size = case["heads"], case["kv_heads"], case["dim"], 2
    if case["op"] == "cache":
        lens = [max(case["new"], n) for n in _lengths(case["seqs"], case["cap"])]
        rows, keys = case["seqs"] * case["new"], sum(lens)
        pairs = sum(case["new"] * n - case["new"] * (case["new"] - 1) // 2 for n in lens)
    else:
        lens = _lengths(case["seqs"], case["most"])
        rows = keys = sum(lens)
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
    q, k = rows * heads * dim * size, keys * kv * dim * size
    if case["op"] == "cache" or not case["train"]:
        return {"bytes": 2 * q + 2 * k + 4 * rows * heads, "flops": 4 * dim * heads * pairs}
    return {"bytes": 4 * q + 4 * k + 4 * rows * heads, "flops": 14 * dim * heads * pairs}


# ---- the definitions in 64 bits, a sequence, a head or a few tokens at a time -----------------------------------------

def _threefry(c0, c1, seed):
    """Threefry-2x32-13 of 32-bit counters held in int64 tensors: both words of each"""
    m = 0xFFFFFFFF
    k = [int(seed) & m, (int(seed) >> 32) & m]
    k.append(k[0] ^ k[1] ^ 0x1BD11BDA)
    turn = [13, 15, 26, 6, 17, 29, 16, 24]
    a, b = (c0 + k[0]) & m, (c1 + k[1]) & m
    for i in range(1, 14):
        a = (a + b) & m
        t = turn[(i - 1) % 8]
        b = (((b << t) & m) | (b >> (32 - t))) ^ a
        if i % 4 == 0:
            a, b = (a + k[(i // 4) % 3]) & m, (b + k[(i // 4 + 1) % 3] + i // 4) & m
    return a, b


def _keep64(index, c0, c1, seed, p):
    """1 / (share kept) or 0, for draws number `index` (0 .. 3) of the counters"""
    a, b = _threefry(c0, c1, seed)
    word = torch.where(index >= 2, b, a)
    low = min(65535, int(round(p * 65536)))
    return torch.where(((word >> (16 * (index % 2))) & 0xFFFF) >= low, 65536.0 / (65536 - low), 0.0).double()


def _exact_dropout(s):
    n = s["X"].numel()
    out = [torch.empty(n, dtype=torch.float64, device="cuda") for _ in range(2)]
    for lo in range(0, n, 1 << 24):
        i = torch.arange(lo, min(n, lo + (1 << 24)), device="cuda")
        keep = _keep64(i % 4, (i // 4) & 0xFFFFFFFF, (i // 4) >> 32, s["seed"], s["drop"])
        part = slice(lo, lo + len(i))
        out[0][part] = s["X"].reshape(-1)[part].double() * keep + s["residual"].reshape(-1)[part].double()
        out[1][part] = s["dY"].reshape(-1)[part].double() * keep
    return tuple(x.reshape(s["X"].shape) for x in out)


def _exact_loss(s):
    W, bias = s["W"].double(), s["bias"].double()
    loss, lse = (torch.zeros(s["tokens"], dtype=torch.float64, device="cuda") for _ in range(2))
    dX, dW, db = torch.zeros(s["X"].shape, dtype=torch.float64, device="cuda"), torch.zeros_like(W), torch.zeros_like(bias)
    for rows in torch.nonzero(s["targets"] >= 0).squeeze(1).split(2048):
        x, t = s["X"][rows].double(), s["targets"][rows]
        z = torch.addmm(bias, x, W.t())
        lse[rows] = torch.logsumexp(z, 1)
        loss[rows] = lse[rows] - z[torch.arange(len(t), device="cuda"), t]
        if s["train"]:
            z = torch.softmax(z, 1)
            z[torch.arange(len(t), device="cuda"), t] -= 1.0
            z *= s["dloss"][rows].double()[:, None]
            dX[rows] = z @ W
            dW += z.t() @ x
            db += z.sum(0)
    return (loss, lse, dX, dW, db) if s["train"] else (loss, lse)


def _exact_attention(s):
    Q, K, V = s["Q"], s["K"], s["V"]
    g = s["heads"] // s["kv_heads"]
    new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse, dQ, dK, dV = new(Q), torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device="cuda"), new(Q), new(K), new(V)
    cu_q, cu_k = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(s["seqs"]):
        q0, q1, k0 = cu_q[b], cu_q[b + 1], cu_k[b]
        k1 = cu_k[b + 1] if s["k_len"] is None else k0 + int(s["k_len"][b])
        if q1 == q0 or k1 == k0:
            continue
        hidden = None
        if s["causal"]:
            hidden = torch.ones(q1 - q0, k1 - k0, dtype=torch.bool, device="cuda").triu((k1 - k0) - (q1 - q0) + 1)
        for h in range(s["heads"]):
            q, k, v = Q[q0:q1, h].double(), K[k0:k1, h // g].double(), V[k0:k1, h // g].double()
            z = q @ k.t() * s["scale"]
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            lse[q0:q1, h] = torch.logsumexp(z, 1)
            w = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
            keep = 1.0
            if s["drop"]:
                j = torch.arange(k1 - k0, device="cuda")
                keep = _keep64(j % 4, torch.arange(q0, q1, device="cuda")[:, None], (1 << 31) + (h << 22) + j // 4, s["seed"], s["drop"])
            out[q0:q1, h] = (w * keep) @ v
            if s["train"]:
                d = s["dO"][q0:q1, h].double()
                dV[k0:k1, h // g] += (w * keep).t() @ d
                dw = (d @ v.t()) * keep
                dz = w * (dw - (w * dw).sum(1, keepdim=True)) * s["scale"]
                dQ[q0:q1, h] = dz @ k
                dK[k0:k1, h // g] += dz.t() @ q
    return (out, lse, dQ, dK, dV) if s["train"] else (out, lse)


def exact(case, seed):
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "loss": _exact_loss}.get(case["op"], _exact_attention)(s)
