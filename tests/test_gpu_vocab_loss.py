"""Cross entropy behind the projection to the vocabulary against the definition in 64 bits, and its gradients.

Tolerances follow from the roundings.  Logits are sums of exact products in 32 bits: 2^-20 of the sum of absolute products covers
their order; loss, lse and dbias inherit that.  d is rounded to bfloat16 (2^-8 of itself) before the products for dX and dW, whose results
are rounded once."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, E32 = 2.0 ** -8, 2.0 ** -20


def say(*a):
    print(*a, flush=True)


class Case:
    def __init__(self, T, V, K, labelled=None, bias=True, std=0.1, seed=1, weights=False):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.X = torch.randn(T, K, generator=g, device=DEV).bfloat16()
        self.W = (torch.randn(V, K, generator=g, device=DEV) * std).bfloat16()
        self.bias = torch.randn(V, generator=g, device=DEV) * 0.3 if bias else None
        labelled = T if labelled is None else labelled
        self.targets = torch.full((T,), -100, dtype=torch.int64, device=DEV)
        at = torch.randperm(T, generator=g, device=DEV)[:labelled]
        self.targets[at] = torch.randint(0, V, (labelled,), generator=g, device=DEV)
        if labelled:
            self.targets[at[0]] = V - 1  # the last word
            self.targets[at[-1]] = 0
        self.dloss = torch.randn(T, generator=g, device=DEV) if weights else torch.full((T,), 1.0 / max(1, labelled), device=DEV)

    def exact(self):
        W = self.W.double()
        X = self.X.double()
        z = X @ W.t() + (self.bias.double() if self.bias is not None else 0.0)
        err = E32 * (X.abs() @ W.abs().t()).amax(1)
        has = (self.targets >= 0) & (self.targets < W.shape[0])
        at = torch.where(has, self.targets, 0)[:, None]
        lse = torch.logsumexp(z, 1)
        loss = lse - z.gather(1, at)[:, 0]
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p).scatter_(1, at, 1.0)
        w = torch.where(has, self.dloss.double(), 0.0)[:, None]
        d = (p - hot) * w
        d_tol = U * d.abs() + (4 * err[:, None] + 1e-6) * p * w.abs() + 2.0 ** -22 * hot * w.abs()
        d_sum = ((4 * err[:, None] + 1e-6) * p * w.abs() + 2.0 ** -20 * (p + hot) * w.abs()).sum(0)
        dX, dW, db = d @ W, d.t() @ X, d.sum(0)
        val = {"loss": torch.where(has, loss, 0.0), "lse": torch.where(has, lse, 0.0), "dX": dX, "dW": dW, "dbias": db}
        tol = {"loss": 2 * err + 1e-6 * (1 + lse.abs() + z.abs().amax(1)), "lse": err + 1e-6 * (1 + lse.abs()),
               "dX": U * dX.abs() + 1.01 * (d_tol @ W.abs()) + 1e-12, "dW": U * dW.abs() + 1.01 * (d_tol.t() @ X.abs()) + 1e-12, "dbias": d_sum + 1e-12}
        return val, tol


def check(name, got, val, tol):
    got = got.double()
    assert torch.isfinite(got).all(), name
    worst = ((got - val).abs() / tol).max().item()
    say("  %s: worst error %.3f of its bound" % (name, worst))
    assert worst <= 1.0, (name, worst)


CASES = {
    "one token, one word": dict(T=1, V=1, K=64),
    "one token": dict(T=1, V=1000, K=128),
    "odd sizes": dict(T=77, V=1003, K=192, labelled=20),
    "words round a tile": dict(T=65, V=257, K=64),
    "no token has a target": dict(T=300, V=500, K=64, labelled=0),
    "all tokens but one": dict(T=300, V=129, K=320, labelled=299),
    "no bias, weights of either sign": dict(T=130, V=600, K=768, bias=False, weights=True),
    "large logits": dict(T=40, V=300, K=256, std=2.0),
    "many tokens": dict(T=1025, V=1001, K=64),
    "many tokens, few targets": dict(T=5000, V=777, K=128, labelled=3),
    "several tiles each way": dict(T=2500, V=2600, K=320, labelled=1111, weights=True),
    "many tokens without a target": dict(T=2000, V=300, K=64, labelled=0),
    "tokens of a whole tile": dict(T=1536, V=512, K=1024, labelled=1280),
}


@pytest.mark.parametrize("name", CASES)
def test_loss_and_gradients(qb, name):
    say("vocabulary loss:", name)
    c = Case(**CASES[name])
    val, tol = c.exact()
    loss, lse = (torch.full(c.targets.shape, float("nan"), device=DEV) for _ in range(2))
    qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias, loss=loss, lse=lse)
    check("loss", loss, val["loss"], tol["loss"])
    check("lse", lse, val["lse"], tol["lse"])
    dX, dW, db = torch.full_like(c.X, float("nan")), torch.full_like(c.W, float("nan")), torch.full((c.W.shape[0],), float("nan"), device=DEV)
    qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias, dX=dX, dW=dW, dbias=db)
    for n, x in (("dX", dX), ("dW", dW), ("dbias", db)):
        check(n, x, val[n], tol[n])
    without = c.targets < 0
    assert (loss[without] == 0).all() and (dX[without] == 0).all()
    again = qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)
    assert torch.equal(again[0], dX) and torch.equal(again[1], dW) and (c.bias is None or torch.equal(again[2], db))


def test_several_pieces_of_the_vocabulary(qb):
    """so many tokens that d of the whole vocabulary is not held at once; few have a target"""
    T, V, K = 300_000, 2000, 64
    say("vocabulary loss in pieces", T, V, K)
    c = Case(T, V, K, labelled=3000)
    loss, lse = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
    dX, dW, db = qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)
    rows = torch.nonzero(c.targets >= 0)[:, 0]
    few = Case(1, 1, 64)
    few.X, few.W, few.bias, few.targets, few.dloss = c.X[rows], c.W, c.bias, c.targets[rows], c.dloss[rows]
    val, tol = few.exact()
    for n, x in (("loss", loss[rows]), ("lse", lse[rows]), ("dX", dX[rows]), ("dW", dW), ("dbias", db)):
        check(n, x, val[n], tol[n])
    assert (dX.abs().sum(1) != 0).sum() == len(rows)


def test_targets_outside_the_vocabulary_have_no_loss(qb):
    c = Case(70, 100, 64)
    want, _ = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets)
    t = c.targets.clone()
    t[::3], t[1::3] = 100, -1
    t[4] = 1 << 40
    got, lse = qb.qb_vocab_loss_fwd(c.X, c.W, t)
    kept = (t >= 0) & (t < 100)
    assert torch.equal(got[kept], want[kept]) and (got[~kept] == 0).all() and (lse[~kept] == 0).all()
    dX, dW, db = qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, t, lse)
    assert db is None and (dX[~kept] == 0).all() and (dX[kept] != 0).any(1).all()


@pytest.mark.parametrize("T", [50, 1100])
def test_gradients_against_differences(qb, T):
    c = Case(T, 333, 128, labelled=T - 9, weights=True)
    loss, lse = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
    grads = dict(zip(("X", "W", "bias"), qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)))
    _, tol = c.exact()
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    for n in ("X", "W", "bias"):
        x = getattr(c, n)
        r = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
        sums = []
        for e in (1e-4, -1e-4):
            setattr(c, n, x.double() + e * r)
            sums.append((c.exact()[0]["loss"] * c.dloss.double()).sum().item())
        setattr(c, n, x)
        slope = (sums[0] - sums[1]) / 2e-4
        bound = (tol["d" + n] * r.abs()).sum().item() + 1e-5 * abs(slope) + 1e-7
        assert abs((grads[n].double() * r).sum().item() - slope) <= bound, n


def test_in_a_graph_and_on_another_stream(qb):
    c = Case(1500, 700, 128, labelled=900)
    want = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
    want += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, want[1], bias=c.bias)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
        got += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, got[1], bias=c.bias)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
        held += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, held[1], bias=c.bias)
    for i in range(4):  # other targets, and other numbers of them
        c.targets[i::5] = -100
        graph.replay()
        torch.cuda.synchronize()
        now = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
        now += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, now[1], bias=c.bias)
        assert all(torch.equal(x, y) for x, y in zip(held, now))


def test_refusals(qb):
    c = Case(20, 50, 64)
    loss, lse = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets)
    with pytest.raises(qb.QBError) as e:
        qb.qb_vocab_loss_fwd(c.X[:, :32].contiguous(), c.W[:, :32].contiguous(), c.targets)
    assert e.value.status == 3
    with pytest.raises(qb.QBError) as e:
        qb.qb_vocab_loss_fwd(c.X[:0], c.W, c.targets[:0])
    assert e.value.status == 3
    with pytest.raises(qb.QBError) as e:
        qb.qb_vocab_loss_fwd(torch.zeros(20 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(20, 64), c.W, c.targets)
    assert e.value.status == 7
    for bad in (lambda: qb.qb_vocab_loss_fwd(c.X.float(), c.W, c.targets), lambda: qb.qb_vocab_loss_fwd(c.X, c.W, c.targets.int()),
                lambda: qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=torch.zeros(50, device=DEV).half()), lambda: qb.qb_vocab_loss_fwd(c.X, c.W.t(), c.targets)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: qb.qb_vocab_loss_fwd(c.X, c.W[:, :32].contiguous(), c.targets), lambda: qb.qb_vocab_loss_fwd(c.X, c.W, c.targets[:-1]),
                lambda: qb.qb_vocab_loss_bwd(c.dloss[:-1], c.X, c.W, c.targets, lse), lambda: qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, dW=c.W[:-1]),
                lambda: qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()


def test_targets_and_bias_from_any_place(qb):
    """A part of a longer tensor of targets (the next words of a text) starts anywhere."""
    c = Case(20, 50, 64)
    inside = lambda x: torch.cat([x[:1], x])[1:]  # noqa: E731
    targets, bias = inside(c.targets), inside(c.bias)
    assert targets.data_ptr() % 16 and bias.data_ptr() % 16
    want = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
    got = qb.qb_vocab_loss_fwd(c.X, c.W, targets, bias=bias)
    want += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, want[1], bias=c.bias)
    got += qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, targets, got[1], bias=bias)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
