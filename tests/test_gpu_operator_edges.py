"""Attention, vocabulary loss and dropout where a call goes to an edge of what its interface allows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


def offsets(*lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("max_q", [0, 500])
def test_sequences_longer_than_named_leave_the_memory_behind_the_workspace(qb, max_q):
    """their results are undefined, but nothing is written beyond the workspace that belongs to the call"""
    say("attention backward, 700 queries where", max_q, "were named")
    import ctypes
    n, heads, dim = 700, 12, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (torch.randn(n, heads, dim, generator=g, device=DEV).bfloat16() for _ in range(4))
    cu = offsets(n)
    O, lse = qb.qb_attention_fwd(q, k, v, cu, cu, n, n)
    a = qb.binding.Attention(Q=q.data_ptr(), K=k.data_ptr(), V=v.data_ptr(), q_row=768, q_head=64, k_row=768, k_head=64, v_row=768, v_head=64, type=0, heads=heads, kv_heads=heads,
                             dim=dim, total_q=n, total_k=n, n_seqs=1, cu_q=cu.data_ptr(), cu_k=cu.data_ptr(), max_q=max_q, max_k=n, scale=0.125)
    room = qb.load_library().qb_attention_bwd_workspace_nbytes(ctypes.byref(a))
    parts = 6 * heads * 2 * 128 * 2 * dim * 4  # of two parts of every tile of keys
    workspace = torch.full((room + parts,), 77, dtype=torch.uint8, device=DEV)
    for x in qb.qb_attention_bwd(do, q, k, v, O, lse, cu, cu, max_q, n, workspace=workspace):
        assert x.shape == q.shape
    assert (workspace[room:] == 77).all()


def test_keys_without_queries_have_no_gradient(qb):
    """no query in the whole tensor, with max_q as an upper bound"""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    q, k, v = (torch.randn(n, 4, 64, generator=g, device=DEV).bfloat16() for n in (0, 100, 100))
    O, lse = qb.qb_attention_fwd(q, k, v, offsets(0, 0), offsets(70, 30), 40, 70)
    grads = [torch.full_like(x, float("nan")) for x in (q, k, v)]
    qb.qb_attention_bwd(q, q, k, v, O, lse, offsets(0, 0), offsets(70, 30), 40, 70, dQ=grads[0], dK=grads[1], dV=grads[2])
    assert O.shape == q.shape and (grads[1] == 0).all() and (grads[2] == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("T,labelled", [(77, 20), (1500, 700), (1500, 1)])
def test_hidden_states_of_tokens_without_a_target_do_not_reach_the_gradients(qb, T, labelled, value):
    say("vocabulary loss, the first and the last token without a target:", T, labelled, value)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    X, W = torch.randn(T, 128, generator=g, device=DEV).bfloat16(), (torch.randn(333, 128, generator=g, device=DEV) * 0.1).bfloat16()
    bias = torch.randn(333, generator=g, device=DEV)
    targets = torch.full((T,), -100, dtype=torch.int64, device=DEV)
    at = 1 + torch.randperm(T - 2, generator=g, device=DEV)[:labelled]
    targets[at] = torch.randint(0, 333, (labelled,), generator=g, device=DEV)
    dloss = torch.full((T,), 1.0 / labelled, device=DEV)

    def outputs():
        loss, lse = qb.qb_vocab_loss_fwd(X, W, targets, bias=bias)
        return (loss, lse) + tuple(qb.qb_vocab_loss_bwd(dloss, X, W, targets, lse, bias=bias))

    want = outputs()
    assert all(torch.isfinite(x).all() for x in want)
    X[0] = X[-1] = value
    assert all(torch.equal(x, y) for x, y in zip(outputs(), want))


@pytest.mark.parametrize("T", [60, 1100])
@pytest.mark.parametrize("power", [127, 100, -100, -126, -130, -149])
def test_weights_of_the_loss_of_any_size(qb, T, power):
    """dloss of a power of two moves the gradients by that power, up to the spacing of the types' least numbers (2^-133, 2^-149)"""
    say("vocabulary loss: gradients of", T, "tokens for a weight of 2 to the", power)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    X, W = torch.randn(T, 128, generator=g, device=DEV).bfloat16(), (torch.randn(333, 128, generator=g, device=DEV) * 0.1).bfloat16()
    targets = torch.randint(0, 333, (T,), generator=g, device=DEV)
    bias = torch.randn(333, generator=g, device=DEV)
    lse = qb.qb_vocab_loss_fwd(X, W, targets, bias=bias)[1]
    weight = torch.ones(T, device=DEV)
    weight[::3] = 0.0
    one = [x.double() * 2.0 ** power for x in qb.qb_vocab_loss_bwd(weight, X, W, targets, lse, bias=bias)]
    got = qb.qb_vocab_loss_bwd(weight * 2.0 ** power, X, W, targets, lse, bias=bias)
    for x, want in zip(got, one):
        over = want.abs() > torch.finfo(x.dtype).max
        assert torch.equal(torch.isfinite(x), ~over)
        least = 2.0 ** -149 if x.dtype == torch.float32 else 2.0 ** -133
        # (below the least normal number a result is rounded a second time here)
        off = (x.double() - want).abs()[~over]
        assert (off <= torch.where(want.abs()[~over] < 2.0 ** -125, 0.51 * least, 0.0)).all()


@pytest.mark.parametrize("name,heads,kv,q_lens,k_lens", [("one launch over a cache", 4, 2, [1, 1, 1], [40, 200, 7]), ("a cache in chunks", 4, 2, [1, 1, 1], [5000, 3000, 7]),
                                                         ("many rows", 24, 24, [300, 257], [300, 400])])
def test_a_query_that_is_no_number_is_not_one_that_sees_no_key(qb, name, heads, kv, q_lens, k_lens):
    say("attention, NaN in a query:", name)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    q, k, v = (torch.randn(sum(n), h, 64, generator=g, device=DEV).bfloat16() for n, h in ((q_lens, heads), (k_lens, kv), (k_lens, kv)))
    call = (k, v, offsets(*q_lens), offsets(*k_lens), max(q_lens), max(k_lens))
    want = qb.qb_attention_fwd(q, *call)
    at = q_lens[0] - 1
    q[at, 1, 3] = float("nan")
    O, lse = qb.qb_attention_fwd(q, *call)
    assert torch.isnan(O[at, 1]).all() and torch.isnan(lse[at, 1])
    dQ, dK, dV = qb.qb_attention_bwd(torch.ones_like(q), q, k, v, O, lse, *call[2:])
    of = 1 // (heads // kv)  # the key head that it reads
    assert torch.isnan(dQ[at, 1]).all() and torch.isnan(dK[0, of]).all() and torch.isnan(dV[0, of]).all()
    assert torch.isfinite(dQ[at, 0]).all() and torch.isfinite(dK[:, -1]).all() and torch.isfinite(dV[:, -1]).all()
    for x, y in ((O, want[0]), (lse, want[1])):
        x[at, 1] = y[at, 1]
        assert torch.equal(x, y)


@pytest.mark.parametrize("T,labelled", [(32768, 700), (32769, 700), (40_000, 1), (70_001, 70_001), (262_145, 3000), (40_000, 0)])
def test_many_tokens_are_numbered_in_order(qb, T, labelled):
    """beyond some tens of thousands the counting of tokens is a launch of its own"""
    from test_gpu_vocab_loss import Case, check
    say("vocabulary loss:", labelled, "of", T, "tokens")
    c = Case(T, 300, 64, labelled=labelled, weights=True)
    c.X[c.targets < 0] = float("nan")
    loss, lse = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias)
    dX, dW, db = qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)
    rows, rest = torch.nonzero(c.targets >= 0)[:, 0], c.targets < 0
    assert (loss[rest] == 0).all() and (lse[rest] == 0).all() and (dX[rest] == 0).all()
    if labelled == 0:
        assert (dW == 0).all() and (db == 0).all()
        return
    few = Case(1, 1, 64)
    few.X, few.W, few.bias, few.targets, few.dloss = c.X[rows], c.W, c.bias, c.targets[rows], c.dloss[rows]
    val, tol = few.exact()
    for n, x in (("loss", loss[rows]), ("lse", lse[rows]), ("dX", dX[rows]), ("dW", dW), ("dbias", db)):
        check(n, x, val[n], tol[n])


def test_the_time_of_many_tokens_grows_with_them(qb):
    """four times the tokens, most of them without a target: not sixteen times the work"""
    def least(T):
        X, W = torch.zeros(T, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(100, 64, dtype=torch.bfloat16, device=DEV)
        targets = torch.full((T,), -100, dtype=torch.int64, device=DEV)
        targets[::100] = 5
        times = []
        for _ in range(5):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            qb.qb_vocab_loss_fwd(X, W, targets)
            end.record()
            torch.cuda.synchronize()
            times.append(begin.elapsed_time(end))
        return min(times)
    few, many = least(1 << 20), least(1 << 22)
    say("vocabulary loss of 2^20 and 2^22 tokens:", few, many, "ms")
    assert many < 8 * few


GUARD = 1 << 16


def guarded(bytes_):
    """a workspace of that size, and whether what lies round it is untouched"""
    held = torch.full((bytes_ + 2 * GUARD,), 77, dtype=torch.uint8, device=DEV)
    return held[GUARD:GUARD + bytes_], lambda: bool((held[:GUARD] == 77).all() and (held[GUARD + bytes_:] == 77).all())


ATTENTION = {
    "one launch over a cache": dict(heads=4, kv_heads=2, q_lens=[1, 2], k_lens=[300, 40], causal=True),
    "a cache in chunks": dict(heads=16, kv_heads=2, q_lens=[5, 1, 0], k_lens=[9000, 700, 40], causal=True),
    "sequences by length": dict(heads=8, kv_heads=8, q_lens=[300, 1, 0, 129, 128, 70]),
    "keys in parts": dict(heads=6, kv_heads=2, q_lens=[2500], causal=True),
    "more keys than queries": dict(heads=3, kv_heads=1, q_lens=[70, 200], k_lens=[3000, 200], causal=True),
    "groups of eighty in parts": dict(heads=80, kv_heads=1, q_lens=[300, 20], k_lens=[300, 400]),
    "many sequences": dict(heads=2, kv_heads=1, q_lens=[(i * 37) % 140 for i in range(70)], p=0.1),
}


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name", ATTENTION)
def test_attention_stays_in_its_workspace(qb, name, dim, type):
    import ctypes
    from test_gpu_attention import Case
    say("attention in a workspace of the size asked for:", name, dim, type)
    c = Case(type, dim, **ATTENTION[name])
    a = ctypes.byref(qb.binding.Attention(Q=c.Q.data_ptr(), K=c.K.data_ptr(), V=c.V.data_ptr(), type=("bf16", "fp16").index(type), heads=c.heads, kv_heads=c.kv, dim=dim, total_q=c.Q.shape[0],
                                          total_k=c.K.shape[0], n_seqs=len(c.q_lens), causal=c.causal, cu_q=c.cu_q.data_ptr(), cu_k=c.cu_k.data_ptr(), max_q=c.max_q, max_k=c.max_k,
                                          scale=c.scale, p=c.p, seed=c.seed.data_ptr() if c.p else None))
    lib = qb.load_library()
    space, untouched = guarded(lib.qb_attention_fwd_workspace_nbytes(a))
    O, lse = c.forward(qb, workspace=space)
    assert untouched()
    space, untouched = guarded(lib.qb_attention_bwd_workspace_nbytes(a))
    grads = c.backward(qb, O, lse, workspace=space)
    assert untouched()
    assert all(torch.equal(x, y) for x, y in zip((O, lse) + tuple(grads), tuple(c.forward(qb)) + tuple(c.backward(qb, O, lse))))


@pytest.mark.parametrize("T,V,K,labelled", [(1, 1, 64, 1), (300, 1003, 128, 300), (512, 30522, 768, 77), (513, 700, 64, 513), (3000, 2600, 320, 1300), (40_000, 3000, 64, 9000), (40_000, 257, 128, 0)])
def test_vocabulary_loss_stays_in_its_workspace(qb, T, V, K, labelled):
    from test_gpu_vocab_loss import Case
    say("vocabulary loss in a workspace of the size asked for:", T, V, K, labelled)
    c, lib = Case(T, V, K, labelled=labelled), qb.load_library()
    space, untouched = guarded(lib.qb_vocab_loss_workspace_nbytes(T, V, K, 0))
    loss, lse = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias, workspace=space)
    assert untouched()
    space, untouched = guarded(lib.qb_vocab_loss_workspace_nbytes(T, V, K, 1))
    grads = qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias, workspace=space)
    assert untouched()
    again = qb.qb_vocab_loss_fwd(c.X, c.W, c.targets, bias=c.bias) + qb.qb_vocab_loss_bwd(c.dloss, c.X, c.W, c.targets, lse, bias=c.bias)
    assert all(torch.equal(x, y) for x, y in zip((loss, lse) + tuple(grads), again))


@pytest.mark.parametrize("low", [float("-inf"), -3.4028234e38])
@pytest.mark.parametrize("T", [70, 700])
def test_words_masked_by_their_bias(qb, T, low):
    """words that nothing may choose, whole tiles of them among those, as padding of the vocabulary has it"""
    say("vocabulary loss: words masked by a bias of", low, T)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    X, W = torch.randn(T, 128, generator=g, device=DEV).bfloat16(), (torch.randn(1500, 128, generator=g, device=DEV) * 0.1).bfloat16()
    bias = torch.full((1500,), low, device=DEV)
    free = torch.cat([torch.arange(3, 200), torch.arange(1290, 1499)]).to(DEV)
    bias[free] = 0.1
    targets = free[torch.randint(0, len(free), (T,), generator=g, device=DEV)]
    dloss = torch.full((T,), 1.0 / T, device=DEV)
    place = torch.full((1500,), -1, device=DEV)
    place[free] = torch.arange(len(free), device=DEV)
    loss, lse = qb.qb_vocab_loss_fwd(X, W, targets, bias=bias)
    want = qb.qb_vocab_loss_fwd(X, W[free], place[targets], bias=bias[free])
    assert all(((x - y).abs() < 1e-5).all() for x, y in zip((loss, lse), want))
    dX, dW, db = qb.qb_vocab_loss_bwd(dloss, X, W, targets, lse, bias=bias)
    dX1, dW1, db1 = qb.qb_vocab_loss_bwd(dloss, X, W[free], place[targets], want[1], bias=bias[free])
    for x, y in ((dX, dX1), (dW[free], dW1), (db[free], db1)):  # (lse and sums in another order: 2^-16, then bfloat16's rounding)
        assert ((x.float() - y.float()).abs() <= 2.0 ** -7 * y.float().abs() + 2.0 ** -16 * y.float().abs().max()).all()
    hidden = torch.ones(1500, dtype=torch.bool, device=DEV)
    hidden[free] = False
    assert (dW[hidden] == 0).all() and (db[hidden] == 0).all()
    targets[5] = 0  # a target that is masked: a loss without bound, a gradient all the same
    loss, lse = qb.qb_vocab_loss_fwd(X, W, targets, bias=bias)
    assert loss[5] > 1e38 and torch.isfinite(loss[:5]).all() and torch.isfinite(lse).all()
    assert all(torch.isfinite(x).all() for x in qb.qb_vocab_loss_bwd(dloss, X, W, targets, lse, bias=bias))


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("max_q,max_k", [(100, 900), (900, 100), (100, 100), (1, 1)])
def test_batches_longer_than_named_stay_in_their_workspace(qb, max_q, max_k, dim, type):
    """sequences in the order of their lengths: workgroups find their tiles by the device's lengths"""
    import ctypes
    from test_gpu_attention import Case
    say("attention of up to 900 queries and keys,", max_q, "and", max_k, "named", dim, type)
    c = Case(type, dim, 8, 8, [900, 100, 640], [700, 900, 640])
    O, lse = c.forward(qb)
    c.max_q, c.max_k = max_q, max_k
    a = ctypes.byref(qb.binding.Attention(Q=c.Q.data_ptr(), K=c.K.data_ptr(), V=c.V.data_ptr(), type=("bf16", "fp16").index(type), heads=8, kv_heads=8, dim=dim, total_q=c.Q.shape[0],
                                          total_k=c.K.shape[0], n_seqs=3, cu_q=c.cu_q.data_ptr(), cu_k=c.cu_k.data_ptr(), max_q=max_q, max_k=max_k, scale=c.scale))
    lib = qb.load_library()
    space, untouched = guarded(lib.qb_attention_fwd_workspace_nbytes(a))
    c.forward(qb, workspace=space)
    assert untouched()
    space, untouched = guarded(lib.qb_attention_bwd_workspace_nbytes(a))
    c.backward(qb, O, lse, workspace=space)
    assert untouched()
