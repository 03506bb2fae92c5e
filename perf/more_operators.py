"""What an encoder layer computes beside its attention when it runs in 16 bits, as timed cases and a generator of more of them.

  norm    layer norm of every token, its backward with the sums over the tokens for weight and bias, and the gradient that comes
          past the norm added on the way; the result also kept in 8 bits for the backward of the linear behind it
  linear  matrix product with bias, activation and residual in one call: a few new tokens, prompts, training steps whose
          backward reads its activations from 8-bit codes (or from 16 bits), and takes the activation's derivative along
  kept    activations written to 8 bits and read back

Where `own` is false, `run` computes them from elementary tensor operations in 32 bits; where it is true, through the
public calls of `paper_1909_05840_amd`.

An activation that is kept in 8 bits is a row of codes -127 .. 127 and one scale for each 64 of its values: the largest magnitude
among them divided by 127 and rounded to 32 bits.  A code is the value divided by the scale, rounded to the nearest whole
number and half to even (0 where the scale is 0), and stands for code times scale.  GELU is z * (1 + erf(z / sqrt 2)) / 2.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GROUP = 64
EPS = 1e-12  # BERT's


def listed():
    return [
        # one new token: the host's call and one launch
        {"name": "norm_1x768_bf16", "op": "norm", "type": "bf16", "tokens": 1, "width": 768, "train": False, "keep": False, "past": False, "wide": False},
        # a large training batch in 16 bits, the residual path's gradient added
        {"name": "norm_train_32768x1024_bf16", "op": "norm", "type": "bf16", "tokens": 32768, "width": 1024, "train": True, "keep": False, "past": True, "wide": False},
        # 32-bit activations as the quantized linears give them, an odd number of tokens and a width that is no multiple of 64
        {"name": "norm_train_6001x1000_fp32", "op": "norm", "type": "fp32", "tokens": 6001, "width": 1000, "train": True, "keep": True, "past": False, "wide": False},
        # one new token through the first linear of a feed-forward block: the weights' bytes
        {"name": "new_1x1024x4096_gelu_bf16", "op": "linear", "type": "bf16", "tokens": 1, "in": 1024, "out": 4096, "act": "gelu", "residual": False, "keep": "no", "train": False,
         "x": "given", "pre": "no", "act_in": "no", "wide": False},
        # the next tokens of 24 requests through the second one
        {"name": "new_24x4096x1024_fp16", "op": "linear", "type": "fp16", "tokens": 24, "in": 4096, "out": 1024, "act": "no", "residual": True, "keep": "no", "train": False,
         "x": "given", "pre": "no", "act_in": "no", "wide": False},
        # an attention block's output projection on one short batch
        {"name": "short_390x768x768_bf16", "op": "linear", "type": "bf16", "tokens": 390, "in": 768, "out": 768, "act": "no", "residual": True, "keep": "no", "train": False,
         "x": "given", "pre": "no", "act_in": "no", "wide": False},
        # long prompts, forward only
        {"name": "prompt_12001x1024x4096_fp16", "op": "linear", "type": "fp16", "tokens": 12001, "in": 1024, "out": 4096, "act": "gelu", "residual": False, "keep": "no", "train": False,
         "x": "given", "pre": "no", "act_in": "no", "wide": False},
        # a training step of a short batch, everything kept in 16 bits
        {"name": "train_390x768x2304_bf16", "op": "linear", "type": "bf16", "tokens": 390, "in": 768, "out": 2304, "act": "no", "residual": False, "keep": "no", "train": True,
         "x": "given", "pre": "no", "act_in": "no", "wide": False},
        # a training step of the first linear: values before GELU kept in 8 bits, its input read back from 8 bits
        {"name": "train_up_16384x1024x4096_bf16", "op": "linear", "type": "bf16", "tokens": 16384, "in": 1024, "out": 4096, "act": "gelu", "residual": False, "keep": "codes", "train": True,
         "x": "kept", "pre": "no", "act_in": "no", "wide": False},
        # a training step of the second: its input is GELU of what the first one kept, and so is the derivative that its backward ends with
        {"name": "train_down_8190x4096x1024_bf16", "op": "linear", "type": "bf16", "tokens": 8190, "in": 4096, "out": 1024, "act": "no", "residual": True, "keep": "no", "train": True,
         "x": "act", "pre": "codes", "act_in": "gelu", "wide": False},
        # activations of one short batch
        {"name": "kept_390x768_fp32", "op": "kept", "type": "fp32", "tokens": 390, "width": 768, "wide": False},
        # of a large one
        {"name": "kept_16384x4096_bf16", "op": "kept", "type": "bf16", "tokens": 16384, "width": 4096, "wide": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "linear", "kept"])
    if op != "linear":
        c = {"op": op, "type": rng.choice(["bf16", "fp16", "fp32"]), "width": _log_int(rng, 8, 4096), "wide": rng.random() < 0.3}
        c["tokens"] = _log_int(rng, 1, min(32768, 32768 * 1024 // c["width"]))
        if op == "norm":
            c["train"] = c["width"] >= 16 and rng.random() < 0.6
            c["keep"], c["past"] = rng.random() < 0.3, c["train"] and rng.random() < 0.5
        return c
    train = rng.random() < 0.5
    c = {"op": op, "type": rng.choice(["bf16", "bf16", "fp16"]), "in": 64 * _log_int(rng, 1, 64), "train": train, "residual": rng.random() < 0.4, "wide": rng.random() < 0.3,
         "act": rng.choice(["no", "gelu", "gelu", "relu", "tanh"]), "keep": "no", "x": "given", "pre": "no", "act_in": "no"}
    c["out"] = rng.choice([64 * rng.randint(1, 64), _log_int(rng, 1, 4096)])
    most = min(16384, 16384 * 1024 * 4096 // (c["in"] * c["out"]))
    c["tokens"] = _log_int(rng, 1, most if train else rng.choice([32, most]))
    if train:
        c["keep"] = rng.choice(["no", "codes", "values"] if c["act"] != "no" else ["no", "codes"])
        c["pre"] = rng.choice(["no", "no", "codes", "values"])
        c["act_in"] = "no" if c["pre"] == "no" else rng.choice(["gelu", "gelu", "relu", "tanh"])
        c["x"] = rng.choice(["given", "kept"] if c["pre"] == "no" else ["given", "act"])
    return c


class _Draw:
    """tensors on the GPU from one seeded generator"""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, type=torch.float32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std).to(type)


def _codes(x):
    """codes [T, W] int8 and scales [T, groups] of x [T, W]"""
    rows, width = x.shape
    groups = -(-width // GROUP)
    x = torch.nn.functional.pad(x.double(), (0, groups * GROUP - width)).reshape(rows, groups, GROUP)
    scales = (x.abs().amax(2) / 127).float()
    by = torch.where(scales > 0, scales, 1.0).double()[..., None]
    return (x / by).round().reshape(rows, -1)[:, :width].to(torch.int8), scales


def _values(codes, scales):
    return codes.float() * scales.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def _part(x, wide):
    """x itself, or the same values as columns of a wider matrix"""
    return torch.nn.functional.pad(x, (8, 16), value=7.0)[:, 8:8 + x.shape[1]] if wide else x


def prepare(case, seed):
    rnd = _Draw(seed)
    s = dict(case)
    t = TYPES[case["type"]]
    if case["op"] != "linear":
        shape = case["tokens"], case["width"]
        # activations have units of their own size and offset, and a few that stand out
        unit = rnd.normal(shape[1], std=0.3).exp_()
        unit[::97] *= 4
        s["X"] = _part((rnd.normal(*shape).mul_(unit) + rnd.normal(shape[1], std=0.3) + 0.2).to(t), case["wide"])
        if case["op"] == "norm":
            s["weight"], s["bias"] = 1 + rnd.normal(shape[1], std=0.1), rnd.normal(shape[1], std=0.1)
            if case["train"]:
                s["dY"] = rnd.normal(*shape, std=1e-2, type=t)
                s["past_grad"] = rnd.normal(*shape, std=1e-2, type=t) if case["past"] else None
        return s
    T, K, N = case["tokens"], case["in"], case["out"]
    s["W"] = rnd.normal(N, K, std=1 / math.sqrt(K), type=t)
    s["bias"] = rnd.normal(N, std=0.1)
    s["residual_in"] = rnd.normal(T, N, type=t) if case["residual"] else None
    X = rnd.normal(T, K, type=t)  # behind a layer norm, or before an activation
    s["kept"] = s["pre_values"] = None
    if case["pre"] != "no":
        s["kept"] = _codes(X) if case["pre"] == "codes" else None
        s["pre_values"] = X if case["pre"] == "values" else None
        X = _ACTS[case["act_in"]](X.float()).to(t)
    elif case["x"] == "kept":
        s["kept"] = _codes(X)
    s["X"] = _part(X, case["wide"])
    if case["train"]:
        s["dY"] = _part(rnd.normal(T, N, std=1e-2, type=t), case["wide"])
    return s


# ---- the plain form: 32 bits, rounded once at the end ---------------------------------------------------------------

def _phi(z):
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


_ACTS = {"no": lambda z: z, "gelu": lambda z: z * _phi(z), "relu": lambda z: z.clamp(min=0), "tanh": torch.tanh}
_SLOPES = {"gelu": lambda z: _phi(z) + z * (-0.5 * z * z).exp() / math.sqrt(2 * math.pi), "relu": lambda z: (z > 0).float(), "tanh": lambda z: 1 - torch.tanh(z) ** 2}


def _plain_kept(s):
    return _values(*_codes(s["X"])).to(s["X"].dtype)


def _plain_norm(s):
    t = s["X"].dtype
    x = s["X"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + EPS).rsqrt()
    hat = d * rstd
    y = hat * s["weight"] + s["bias"]
    out = [y.to(t), mean.squeeze(1), rstd.squeeze(1)]
    if s["keep"]:
        out.append(_values(*_codes(y)).to(torch.bfloat16))
    if s["train"]:
        dy = s["dY"].float()
        g = dy * s["weight"]
        dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
        if s["past"]:
            dx = dx + s["past_grad"].float()
        out += [dx.to(t), (dy * hat).sum(0), dy.sum(0)]
    return out


def _plain_linear(s):
    t = s["X"].dtype
    W = s["W"].float()
    z = s["X"].float() @ W.t() + s["bias"]
    y = _ACTS[s["act"]](z)
    if s["residual"]:
        y = y + s["residual_in"].float()
    out = [y.to(t)]
    if s["keep"] == "codes":
        out.append(_values(*_codes(y if s["act"] == "no" else z)).to(t))
    elif s["keep"] == "values":
        out.append(z.to(t))
    if s["train"]:
        dy = s["dY"].float()
        dx, x = dy @ W, s["X"].float()
        if s["kept"] is not None:
            x = _values(*s["kept"])
        if s["pre"] != "no":
            pre = x if s["pre"] == "codes" else s["pre_values"].float()
            dx = dx * _SLOPES[s["act_in"]](pre)
            x = _ACTS[s["act_in"]](pre) if s["x"] == "act" else s["X"].float()
        out += [dx.to(t), (dy.t() @ x).to(t), dy.sum(0)]
    return out


def run(s):
    op = s["op"]
    if not own:
        return _plain_kept(s) if op == "kept" else _plain_norm(s) if op == "norm" else _plain_linear(s)
    import paper_1909_05840_amd as qb
    X, t = s["X"], s["X"].dtype
    if op == "kept":
        return qb.qb_restore_act(*qb.qb_checkpoint_act(X), t)
    if op == "norm":
        out = list(qb.qb_layer_norm_fwd(X, s["weight"], s["bias"], EPS, keep=s["keep"]))
        if s["keep"]:
            out[3:] = [qb.qb_restore_act(*out[3:], torch.bfloat16)]
        if s["train"]:
            out += qb.qb_layer_norm_bwd(s["dY"], X, s["weight"], out[1], out[2], residual=s["past_grad"])
        return out
    act = lambda name: None if name == "no" else name  # noqa: E731
    got = qb.qb_linear_fwd(X, s["W"], s["bias"], act=act(s["act"]), residual=s["residual_in"], keep=None if s["keep"] == "no" else s["keep"])
    out = [got[0], qb.qb_restore_act(*got[1], t)] if s["keep"] == "codes" else list(got) if s["keep"] == "values" else [got]
    if s["train"]:
        pre = s["kept"] if s["pre"] == "codes" else s["pre_values"]
        out += qb.qb_linear_bwd(s["dY"], s["kept"] if s["x"] == "kept" else None if s["x"] == "act" else X, s["W"], pre=pre, act=act(s["act_in"]))
    return out


def work(case):
    size = TYPES[case["type"]].itemsize
    T = case["tokens"]
    if case["op"] != "linear":
        values = T * case["width"]
        codes = values + 4 * T * -(-case["width"] // GROUP)
        if case["op"] == "kept":
            return {"bytes": 2 * values * size + 2 * codes, "flops": 0}
        b = 2 * values * size + 8 * T + 8 * case["width"] + (codes + 2 * values if case["keep"] else 0)
        if case["train"]:
            b += (3 + case["past"]) * values * size + 8 * T + 12 * case["width"]
        return {"bytes": b, "flops": 0}
    K, N = case["in"], case["out"]
    x, w, y = T * K * size, N * K * size, T * N * size
    b = x + w + 4 * N + y * (2 if case["residual"] else 1)
    b += T * N * (1 + size) if case["keep"] == "codes" else y if case["keep"] == "values" else 0
    if not case["train"]:
        return {"bytes": b, "flops": 2 * T * N * K}
    # dY, W and the kept input in, dX, dW and the bias's gradient out
    b += y + w + x + w + 4 * N
    b += T * K if case["x"] == "kept" or case["pre"] == "codes" else 0
    b += x if case["pre"] == "values" else 0
    b += x if case["x"] == "given" else 0
    return {"bytes": b, "flops": 6 * T * N * K}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _nearest64(x):
    """what 8 bits keep of x, a group of columns at a time"""
    out = torch.zeros_like(x)
    for at in range(0, x.shape[1], GROUP):
        g = x[:, at:at + GROUP]
        scale = (g.abs().max(1, keepdim=True).values / 127.0).to(torch.float32).to(torch.float64)
        out[:, at:at + GROUP] = torch.where(scale == 0, 0.0, torch.round(g / scale) * scale)
    return out


def _act64(name, z):
    """an activation and its derivative"""
    if name == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    if name == "tanh":
        return torch.tanh(z), 1 / torch.cosh(z) ** 2
    if name == "gelu":
        share = torch.special.erfc(-z / math.sqrt(2.0)) / 2
        return z * share, share + z * torch.exp(-z * z / 2) / math.sqrt(2.0 * math.pi)
    return z, torch.ones_like(z)


def _exact_norm(s):
    x, w, b = s["X"].double(), s["weight"].double(), s["bias"].double()
    width = x.shape[1]
    mean = x.sum(1) / width
    var = ((x - mean[:, None]) ** 2).sum(1) / width
    rstd = 1 / torch.sqrt(var + EPS)
    hat = (x - mean[:, None]) * rstd[:, None]
    y = hat * w + b
    out = [y, mean, rstd]
    if s["keep"]:
        out.append(_nearest64(y))
    if s["train"]:
        dy = s["dY"].double()
        g = dy * w
        dx = (g - (g.sum(1, keepdim=True) + hat * (g * hat).sum(1, keepdim=True)) / width) * rstd[:, None]
        out += [dx + s["past_grad"].double() if s["past"] else dx, (dy * hat).sum(0), dy.sum(0)]
    return out


def _exact_linear(s):
    X, W = s["X"].double(), s["W"].double()
    z = torch.addmm(s["bias"].double(), X, W.t())
    y = _act64(s["act"], z)[0]
    if s["residual"]:
        y = y + s["residual_in"].double()
    out = [y]
    if s["keep"] != "no":
        out.append(z if s["keep"] == "values" else _nearest64(y if s["act"] == "no" else z))
    if s["train"]:
        dy = s["dY"].double()
        dx = dy @ W
        back = None
        if s["kept"] is not None:
            codes, scales = s["kept"]
            back = codes.double()
            for g in range(scales.shape[1]):
                back[:, g * GROUP:(g + 1) * GROUP] *= scales[:, g:g + 1].double()
        if s["pre"] != "no":
            value, slope = _act64(s["act_in"], back if s["pre"] == "codes" else s["pre_values"].double())
            dx = dx * slope
            X = value if s["x"] == "act" else X
        elif s["x"] == "kept":
            X = back
        out += [dx, dy.t() @ X, dy.sum(0)]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "kept":
        return _nearest64(s["X"].double())
    return _exact_norm(s) if case["op"] == "norm" else _exact_linear(s)
