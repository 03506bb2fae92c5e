"""Activations in 8 bits: codes and scales bit for bit, what they stand for, rows apart, short groups, ties, extremes."""
import math

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,W", [(1, 1), (1, 64), (3, 65), (7, 63), (2, 128), (390, 768), (33, 1000), (5, 4097), (1025, 72), (2, 32768)])
def test_bit_for_bit(qb, t, T, W):
    X = ref.draw(T, W, seed=T * W, t=t)
    codes, scales = qb.qb_checkpoint_act(X.cuda())
    want = ref.keep(X)
    assert torch.equal(codes.cpu(), want[0]) and torch.equal(scales.cpu(), want[1])
    for out in TYPES:
        assert torch.equal(qb.qb_restore_act(codes, scales, out).cpu(), ref.restore(*want).float().to(out))


def test_ties_go_to_the_even_code(qb):
    # a scale of one: the quotients are the values themselves, halves among them, and the two neighbours of each half
    half = torch.arange(-126, 126, dtype=torch.float64) + 0.5
    up, down = torch.nextafter(half.float(), torch.tensor(math.inf)), torch.nextafter(half.float(), torch.tensor(-math.inf))
    x = torch.cat([half.float(), up, down])
    x = torch.cat([torch.full((12, 1), 127.0), x.reshape(12, 63)], 1)
    codes, scales = qb.qb_checkpoint_act(x.cuda())
    assert (scales == 1).all()
    assert torch.equal(codes.cpu().double(), torch.round(x.double()))


def test_quotients_next_to_a_half(qb):
    # values that the rounded reciprocal alone would put on the wrong side: x is the value nearest to (k + 1/2) scale, and its neighbours
    g = torch.Generator().manual_seed(3)
    top = torch.rand(4000, generator=g) * 100 + 0.01
    scale = (top.double() / 127).float().double()
    k = torch.randint(0, 126, (4000, 20), generator=g)
    near = ((k + 0.5) * scale[:, None]).float()
    x = torch.cat([top[:, None], near, torch.nextafter(near, torch.tensor(math.inf)), -torch.nextafter(near, torch.tensor(0.0))], 1)
    want = ref.keep(x)
    codes, scales = qb.qb_checkpoint_act(x.cuda())
    assert torch.equal(scales.cpu(), want[1]) and torch.equal(codes.cpu(), want[0])


def test_rows_apart_and_given_outputs(qb):
    wide = ref.draw(37, 300, seed=5, t=torch.bfloat16).cuda()
    for a, b in ((0, 200), (1, 130), (173, 300)):
        codes = torch.full((37, b - a), 77, dtype=torch.int8, device="cuda")
        got = qb.qb_checkpoint_act(wide[:, a:b], codes=codes)
        want = ref.keep(wide[:, a:b].cpu())
        assert got[0].data_ptr() == codes.data_ptr()
        assert torch.equal(codes.cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])
    row = wide[:1].expand(9, 300)  # the same row nine times
    assert torch.equal(qb.qb_checkpoint_act(row)[0].cpu(), ref.keep(row.cpu())[0])


def test_nothing_behind_the_outputs_is_written(qb):
    for T, W in ((3, 65), (1, 1), (5, 127)):
        room = torch.full((T * W + 64,), 55, dtype=torch.int8, device="cuda")
        scale_room = torch.full((T * -(-W // 64) + 16,), 9.0, device="cuda")
        back = torch.full((T * W + 64,), 3.0, dtype=torch.float16, device="cuda")
        X = ref.draw(T, W, seed=1, t=torch.float32).cuda()
        codes, scales = qb.qb_checkpoint_act(X, codes=room[:T * W].view(T, W), scales=scale_room[:T * -(-W // 64)].view(T, -1))
        qb.qb_restore_act(codes, scales, X=back[:T * W].view(T, W))
        assert (room[T * W:] == 55).all() and (scale_room[scales.numel():] == 9).all() and (back[T * W:] == 3).all()


def test_extremes(qb):
    x = torch.zeros(6, 64)
    x[1] = 1e-45             # a scale that rounds to zero
    x[2, 3] = torch.finfo(torch.float32).max
    x[2, 4] = -1.0
    x[3] = 190 * 1.401298464e-45  # subnormal scale: the quotient is beyond 127
    x[4, 0], x[4, 1] = math.inf, 2.0
    x[5, 7], x[5, 8] = math.nan, 2.0
    codes, scales = (v.cpu() for v in qb.qb_checkpoint_act(x.cuda()))
    want = ref.keep(x[:4])
    assert torch.equal(codes[:4], want[0]) and torch.equal(scales[:4], want[1])
    assert (codes[0] == 0).all() and scales[0, 0] == 0 and codes[2, 3] == 127 and (codes[3] == 127).all()
    back = qb.qb_restore_act(codes.cuda(), scales.cuda(), torch.float32).cpu()
    assert back[4:].isnan().all() and not back[:4].isnan().any()


def test_no_rows(qb):
    codes, scales = qb.qb_checkpoint_act(torch.empty(0, 100, device="cuda"))
    assert codes.shape == (0, 100) and scales.shape == (0, 2)
    assert qb.qb_restore_act(codes, scales, torch.float16).shape == (0, 100)


def test_another_stream_and_a_graph(qb):
    X = ref.draw(700, 777, seed=2, t=torch.float16).cuda()
    want = ref.keep(X.cpu())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        codes, scales = qb.qb_checkpoint_act(X)
    side.synchronize()
    assert torch.equal(codes.cpu(), want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, s = qb.qb_checkpoint_act(X)
        back = qb.qb_restore_act(c, s, torch.float16)
    for seed in range(3):
        X.copy_(ref.draw(700, 777, seed=10 + seed, t=torch.float16))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.keep(X.cpu())
        assert torch.equal(c.cpu(), want[0]) and torch.equal(s.cpu(), want[1])
        assert torch.equal(back.cpu(), ref.restore(*want).float().to(torch.float16))
