"""Dropout from a counter-based generator against its definition in whole numbers and 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def draws(n, seed):
    """16-bit draws 0 .. n-1: Threefry-2x32, 13 rounds, four draws a counter"""
    m = 0xFFFFFFFF
    k = [seed & m, (seed >> 32) & m]
    k.append(k[0] ^ k[1] ^ 0x1BD11BDA)
    i = torch.arange(n, device=DEV)
    c = i // 4
    a, b = ((c & m) + k[0]) & m, ((c >> 32) + k[1]) & m
    for r in range(13):
        a = (a + b) & m
        t = (13, 15, 26, 6, 17, 29, 16, 24)[r % 8]
        b = (((b << t) & m) | (b >> (32 - t))) ^ a
        if r % 4 == 3:
            j = r // 4 + 1
            a, b = (a + k[j % 3]) & m, (b + k[(j + 1) % 3] + j) & m
    return (torch.where(i % 4 >= 2, b, a) >> (16 * (i % 2))) & 0xFFFF


def keep64(n, p, seed):
    t = min(65535, round(p * 65536))
    return (draws(n, seed) >= t).double() * (65536.0 / (65536 - t))


def near(got, want, u, off=0.0):
    """got is want within one rounding to its type and `off`: u of itself, the spacing of the least numbers below those (2^-25 half of
    float16's), infinity beyond its largest"""
    over = torch.isinf(want.to(got.dtype))
    least = 2.0 ** -25 if got.dtype == torch.float16 else 0.0
    return torch.where(over, got.double() == want.to(got.dtype).double(), (got.double() - want).abs() <= u * want.abs() + off + least).all()


def seed_tensor(v):
    return torch.tensor([v], dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 63, 255, 1023, 1025, 4099, 2_000_003])
def test_values_and_gradients(qb, type, n):
    print("dropout", type, n, flush=True)
    dtype, u = TYPES[type]
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    X, R, dY = (torch.randn(n, generator=g, device=DEV).to(dtype) for _ in range(3))
    for p, s in ((0.1, 77 - n), (0.5, -(1 << 62)), (0.0, 5), (0.99999, (1 << 62) + 9)):
        keep, seed = keep64(n, p, s), seed_tensor(s)
        # a product and a sum in 32 bits (the scale is itself rounded), then the type's rounding
        want = X.double() * keep + R.double()
        assert near(qb.qb_dropout_fwd(X, p, seed, residual=R), want, u, 2.0 ** -22 * ((X.double() * keep).abs() + R.double().abs()))
        y, want = qb.qb_dropout_fwd(X, p, seed), X.double() * keep
        assert near(y, want, u + 2.0 ** -22) and (y[keep == 0] == 0).all()
        assert near(qb.qb_dropout_bwd(dY, p, seed), dY.double() * keep, u + 2.0 ** -22)


def test_gradient_against_differences(qb):
    n, p, seed = 4097, 0.3, seed_tensor(12345)
    X = torch.linspace(-2, 2, n, device=DEV)
    dY = torch.linspace(1, 3, n, device=DEV)
    dX = qb.qb_dropout_bwd(dY, p, seed)
    e = 0.5  # (linear: any step will do, and this one is exact in the inputs' exponents up to a rounding)
    up, down = qb.qb_dropout_fwd(X + e, p, seed), qb.qb_dropout_fwd(X - e, p, seed)
    slope = (up.double() - down.double()) / ((X + e).double() - (X - e).double()) * dY.double()
    assert ((dX.double() - slope).abs() <= 1e-5 * (1 + dX.double().abs())).all()


@pytest.mark.parametrize("type", TYPES)
def test_addresses_of_any_kind_and_in_place(qb, type):
    """the values do not depend on where the tensors lie; outputs may take the place of inputs"""
    dtype, _ = TYPES[type]
    n, seed = 5003, seed_tensor(99)
    X, R = torch.randn(n, device=DEV).to(dtype), torch.randn(n, device=DEV).to(dtype)
    want, plain = qb.qb_dropout_fwd(X, 0.1, seed, residual=R), qb.qb_dropout_fwd(X, 0.1, seed)
    for a, b, c in ((0, 0, 1), (1, 0, 0), (0, 3, 0), (5, 2, 7), (4, 4, 4), (8, 8, 8)):
        held = torch.full((3, n + 16), 3.0, dtype=dtype, device=DEV).reshape(-1)
        x, r, y = held[a:a + n], held[n + 16 + b:2 * n + 16 + b], held[2 * n + 32 + c:3 * n + 32 + c]
        x.copy_(X)
        r.copy_(R)
        qb.qb_dropout_fwd(x, 0.1, seed, residual=r, Y=y)
        assert torch.equal(y, want)
        assert held[2 * n + 32 + c - 1] == 3.0 and held[3 * n + 32 + c] == 3.0
        qb.qb_dropout_fwd(x, 0.1, seed, residual=r, Y=r)
        assert torch.equal(r, want)
        qb.qb_dropout_fwd(x, 0.1, seed, Y=x)
        assert torch.equal(x, plain)


def test_share_dropped_and_seeds(qb):
    n = 1 << 22
    X = torch.ones(n, device=DEV)
    seen = []
    for s in (1, 2, 1 << 32, -1):
        for p in (0.05, 0.1, 0.5):
            share = (qb.qb_dropout_fwd(X, p, seed_tensor(s)) == 0).double().mean().item()
            assert abs(share - p) < 6 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17
        seen.append(qb.qb_dropout_fwd(X, 0.5, seed_tensor(s)) == 0)
    for i in range(len(seen)):
        for j in range(i):  # independent masks of one half agree on half of the values
            assert abs((seen[i] == seen[j]).double().mean().item() - 0.5) < 6 * 0.5 / n ** 0.5
        assert abs((seen[i][1:] == seen[i][:-1]).double().mean().item() - 0.5) < 6 * 0.5 / n ** 0.5


def test_empty_and_refusals(qb):
    x, s = torch.ones(8, device=DEV), seed_tensor(1)
    assert qb.qb_dropout_fwd(x[:0], 0.1, s).numel() == 0
    for p in (1.0, -0.1, float("nan"), float("inf")):
        with pytest.raises(qb.QBError) as e:
            qb.qb_dropout_fwd(x, p, s)
        assert e.value.status == 7
    with pytest.raises(qb.QBError):
        qb.qb_dropout_fwd(x, 0.1, None)
    for bad in (lambda: qb.qb_dropout_fwd(x.double(), 0.1, s), lambda: qb.qb_dropout_fwd(x, 0.1, s.int()), lambda: qb.qb_dropout_fwd(x, 0.1, s, residual=x.half()),
                lambda: qb.qb_dropout_fwd(x[::2], 0.1, s), lambda: qb.qb_dropout_bwd(x, 0.1, s, dX=x.half()), lambda: qb.qb_dropout_fwd(x.cpu(), 0.1, s)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: qb.qb_dropout_fwd(x, 0.1, torch.ones(2, dtype=torch.int64, device=DEV)), lambda: qb.qb_dropout_fwd(x, 0.1, s, residual=x[:4])):
        with pytest.raises(ValueError):
            bad()
