"""Layer norm, linears and 8-bit activations in 64 bits, for the tests of these operators, and the roundings that their results may be off by."""
import math

import torch

GROUP = 64
STEP = 2.0 ** -24          # half a step of binary32, relative
NORMAL = 2.0 ** -15        # what the kernels' normal distribution is off, relative to its smaller tail


def half_step(t):
    return torch.finfo(t).eps / 2


def draw(*shape, seed, std=1.0, mean=0.0, t=torch.float64):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std + mean).to(t)


def groups_of(x):
    """[rows, groups, 64], zeros behind the last column"""
    rows, width = x.shape
    n = -(-width // GROUP)
    return torch.nn.functional.pad(x, (0, n * GROUP - width)).reshape(rows, n, GROUP)


def keep(x):
    """codes and scales by the definition, in 64 bits from exact values"""
    g = groups_of(x.double())
    scales = (g.abs().amax(2) / 127).float()
    s = scales.double()[..., None]
    codes = torch.where(s > 0, torch.round(g / torch.where(s > 0, s, 1.0)), 0.0).clamp(-127, 127)
    return codes.reshape(len(x), -1)[:, :x.shape[1]].to(torch.int8), scales


def restore(codes, scales):
    return codes.double() * scales.double().repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def check_kept(codes, scales, z, off):
    """Codes and scales of values that are within `off` of z: the scale is that of the largest magnitude, the values are within half a scale."""
    codes, scales = codes.cpu(), scales.cpu()
    top, slack = groups_of(z).abs().amax(2), groups_of(off).amax(2)
    assert ((scales.double() * 127 - top).abs() <= slack + 2 * STEP * top).all()
    half = scales.double().repeat_interleave(GROUP, 1)[:, :z.shape[1]] * (0.5 + 2.0 ** -16)
    assert ((restore(codes, scales) - z).abs() <= half + off).all()
    assert (codes >= -127).all()


def phi(z):
    return torch.special.erfc(-z / math.sqrt(2)) / 2


def act(name, z):
    """an activation, its derivative, and what the kernels' own arithmetic may make either off"""
    one = torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), 0 * z, 0 * z
    if name == "tanh":
        t = torch.tanh(z)
        return t, 1 / torch.cosh(z) ** 2, 16 * STEP * t.abs(), 32 * STEP * one
    if name == "gelu":
        p, bell = phi(z), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        tail = torch.minimum(p, 1 - p)
        return z * p, p + z * bell, (NORMAL * tail + 16 * STEP) * z.abs(), NORMAL * tail + 32 * STEP * (1 + z.abs())
    return z, one, 0 * z, 0 * z


def near(got, want, off, what):
    got = got.cpu().double()
    bad = ~((got - want).abs() <= off)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g over its bound %.3g" % (
        what, int(bad.sum()), bad.numel(), ((got - want).abs() - off).nan_to_num(nan=math.inf).max(), off[bad].max())
