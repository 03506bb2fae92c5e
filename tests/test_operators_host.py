"""Dropout, attention and vocabulary loss on the host: workspace sizes, and every refusal comes before a launch (no GPU needed)."""
import ctypes

import pytest

import paper_1909_05840_amd as qb

P, AT16, AT4, ODD = 0x1000, 0x1010, 0x1004, 0x1001  # addresses that are checked and never read
BF16, FP16, FP32 = 0, 1, 2
NULL, SHAPE, VALUE, WORKSPACE = 1, 3, 7, 5
f = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    return qb.load_library()


def attention(**changed):
    """Four sequences of up to 40 in 100 rows; 12 heads of 64 side by side in rows of queries, keys and values."""
    a = dict(Q=P, K=P, V=P, q_row=2304, q_head=64, k_row=2304, k_head=64, v_row=2304, v_head=64, type=BF16, heads=12, kv_heads=12, dim=64,
             total_q=100, total_k=100, n_seqs=4, causal=0, cu_q=P, cu_k=P, k_len=None, max_q=40, max_k=40, scale=0.125, p=0.0, seed=None)
    a.update(changed)
    return ctypes.byref(qb.binding.Attention(**a))


def grads(**changed):
    g = dict(dQ=P, dK=P, dV=P, q_row=2304, q_head=64, k_row=2304, k_head=64, v_row=2304, v_head=64)
    g.update(changed)
    return ctypes.byref(qb.binding.AttentionGrads(**g))


def test_status_has_a_text():
    assert qb.qb_status_string(VALUE) not in ("", qb.qb_status_string(99))


REFUSED = [
    (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL), (dict(cu_q=None), NULL), (dict(cu_k=None), NULL),
    (dict(p=0.1), NULL),  # no seed
    (dict(dim=96), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=5), SHAPE), (dict(total_q=-1), SHAPE),
    (dict(total_k=-1), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_k=-1), SHAPE), (dict(total_q=2 ** 31), SHAPE),
    (dict(total_k=2 ** 31), SHAPE), (dict(max_q=2 ** 30), SHAPE), (dict(max_k=2 ** 31), SHAPE),
    (dict(p=0.1, seed=P, heads=1024, kv_heads=1024), SHAPE), (dict(p=0.1, seed=P, max_k=2 ** 24 + 1), SHAPE),
    (dict(type=FP32), VALUE), (dict(type=-1), VALUE), (dict(scale=0.0), VALUE), (dict(scale=-1.0), VALUE), (dict(scale=float("nan")), VALUE),
    (dict(scale=float("inf")), VALUE), (dict(p=1.0, seed=P), VALUE), (dict(p=-0.1, seed=P), VALUE), (dict(p=float("nan"), seed=P), VALUE),
    (dict(q_row=2305), VALUE), (dict(k_head=68), VALUE), (dict(v_row=4), VALUE), (dict(Q=0x1002), VALUE), (dict(K=0x1008), VALUE), (dict(V=ODD), VALUE),
]


@pytest.mark.parametrize("changed, status", REFUSED)
def test_attention_refuses(lib, changed, status):
    assert lib.qb_attention_fwd(attention(**changed), P, P, P, None) == status
    assert lib.qb_attention_bwd(attention(**changed), P, P, P, grads(), P, None) == status


def test_attention_refuses_outputs(lib):
    a = attention()
    assert lib.qb_attention_fwd(None, P, P, P, None) == NULL
    assert lib.qb_attention_fwd(a, None, P, P, None) == NULL
    assert lib.qb_attention_fwd(a, P, None, P, None) == NULL
    assert lib.qb_attention_fwd(a, 0x1008, P, P, None) == VALUE
    assert lib.qb_attention_bwd(a, P, P, P, None, P, None) == NULL
    for at in range(3):  # dO, O, lse
        assert lib.qb_attention_bwd(a, *(None if i == at else P for i in range(3)), grads(), P, None) == NULL
    for name in ("dQ", "dK", "dV"):
        assert lib.qb_attention_bwd(a, P, P, P, grads(**{name: None}), P, None) == NULL
        assert lib.qb_attention_bwd(a, P, P, P, grads(**{name: 0x1008}), P, None) == VALUE
    assert lib.qb_attention_bwd(a, P, P, P, grads(q_row=2308), P, None) == VALUE
    assert lib.qb_attention_bwd(a, P, P, P, grads(), None, None) == WORKSPACE
    assert lib.qb_attention_bwd(a, P, P, P, grads(), AT16, None) == WORKSPACE
    assert lib.qb_attention_bwd(attention(k_len=P), P, P, P, grads(), P, None) == VALUE  # a cache has no backward
    cache = attention(total_q=4, max_q=1, k_len=P, total_k=1 << 18, max_k=1 << 16, kv_heads=4)
    assert lib.qb_attention_fwd_workspace_nbytes(cache) > 0  # long keys of few rows are shared out
    assert lib.qb_attention_fwd(cache, P, P, None, None) == WORKSPACE
    assert lib.qb_attention_fwd(cache, P, P, AT16, None) == WORKSPACE


def test_attention_with_nothing_to_do(lib):
    assert lib.qb_attention_fwd(attention(total_q=0, Q=None), None, None, None, None) == 0
    assert lib.qb_attention_fwd(attention(n_seqs=0, cu_q=None, cu_k=None), None, None, None, None) == 0
    assert lib.qb_attention_bwd(attention(total_q=0, total_k=0, Q=None, K=None, V=None), None, None, None, grads(dQ=None, dK=None, dV=None), None, None) == 0


def test_attention_workspaces(lib):
    assert lib.qb_attention_fwd_workspace_nbytes(attention()) == 0
    assert lib.qb_attention_bwd_workspace_nbytes(attention()) >= 2 * (100 * 12 + 1) * 4  # two statistics a row
    assert lib.qb_attention_bwd_workspace_nbytes(attention(total_q=2 ** 24)) >= 2 * (2 ** 24 * 12 + 1) * 4
    for bad in (dict(dim=80), dict(heads=-1), dict(type=9)):
        assert lib.qb_attention_fwd_workspace_nbytes(attention(**bad)) == 0
        assert lib.qb_attention_bwd_workspace_nbytes(attention(**bad)) == 0


def test_dropout_refuses(lib):
    for call in (lambda X, n, t, p, s, Y: lib.qb_dropout_fwd(X, None, n, t, f(p), s, Y, None), lambda X, n, t, p, s, Y: lib.qb_dropout_bwd(X, n, t, f(p), s, Y, None)):
        assert call(None, 8, BF16, 0.1, P, P) == NULL
        assert call(P, 8, BF16, 0.1, None, P) == NULL
        assert call(P, 8, BF16, 0.1, P, None) == NULL
        assert call(P, -1, BF16, 0.1, P, P) == SHAPE
        for p in (1.0, -0.1, float("nan"), float("inf")):
            assert call(P, 8, BF16, p, P, P) == VALUE
        assert call(P, 8, 3, 0.1, P, P) == VALUE
        assert call(ODD, 8, FP16, 0.1, P, P) == VALUE
        assert call(P, 8, FP32, 0.1, P, 0x1002) == VALUE
        assert call(P, 8, FP32, 0.1, AT4, P) == VALUE  # a seed of eight bytes
        assert call(None, 0, FP32, 0.1, None, None) == 0
    assert lib.qb_dropout_fwd(P, 0x1002, 8, FP32, f(0.1), P, P, None) == VALUE


def test_vocab_loss_refuses(lib):
    def fwd(X=P, W=P, bias=P, targets=P, T=10, V=100, K=128, loss=P, lse=P, workspace=P):
        return lib.qb_vocab_loss_fwd(X, W, bias, targets, T, V, K, loss, lse, workspace, None)

    def bwd(dloss=P, X=P, W=P, bias=P, targets=P, lse=P, T=10, V=100, K=128, dX=P, dW=P, dbias=P, workspace=P):
        return lib.qb_vocab_loss_bwd(dloss, X, W, bias, targets, lse, T, V, K, dX, dW, dbias, workspace, None)

    for call, names in ((fwd, ("X", "W", "targets", "loss", "lse")), (bwd, ("dloss", "X", "W", "targets", "lse", "dX", "dW"))):
        for name in names:
            assert call(**{name: None}) == NULL, name
        for bad in (dict(T=0), dict(T=-1), dict(T=2 ** 24 + 1), dict(V=0), dict(V=2 ** 24 + 1), dict(K=0), dict(K=100), dict(K=2 ** 20)):
            assert call(**bad) == SHAPE, bad
        for bad in (dict(X=0x1008), dict(W=0x1002), dict(targets=AT4)):
            assert call(**bad) == VALUE, bad
        assert call(workspace=None) == WORKSPACE
        assert call(workspace=AT16) == WORKSPACE
    assert bwd(dX=0x1008) == VALUE and bwd(dW=0x1008) == VALUE


def test_vocab_loss_workspaces(lib):
    size = lib.qb_vocab_loss_workspace_nbytes
    assert 0 < size(390, 30522, 768, 0) < size(390, 30522, 768, 1)
    # the gradient of the logits is worked off in pieces: its share does not grow past one of them
    assert size(65536, 128000, 1024, 1) < 65536 * 128000 * 2
    for bad in ((0, 100, 128), (10, 0, 128), (10, 100, 100), (2 ** 24 + 1, 100, 128)):
        assert size(*bad, 0) == 0 and size(*bad, 1) == 0
