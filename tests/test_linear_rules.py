"""The 16-bit linears' rules for tiles and for parts of their contractions, on the host (no GPU needed)."""
import ctypes

import pytest

from linear_plans import BACKWARD, FORWARD, NEEDS
from paper_1909_05840_amd.binding import LIB_PATH, LinearGrads, LinearLayer, load_library

P = 0x1000  # an address that is checked and never read


def linear(T, N, K, codes=False):
    return ctypes.byref(LinearLayer(type=0, act=0, T=T, N=N, K=K, X=P, x_row=K, W=P, Y=P, codes=P if codes else None, scales=P if codes else None))


# One output, us, cut (as if a part's row were as short as the result's) and as 64 outputs are: 20000 x 1 by 768 15.5, 7.7; 8278 x 1 by 2240 15.8, 11.9; 20000 x 1 by 4096 32.4, 26.8
@pytest.mark.parametrize("T", [100, 300, 1000, 3000, 8278, 20000, 100000])
@pytest.mark.parametrize("K", [768, 1024, 2240, 4096])
def test_narrow_results_are_cut_as_whole_groups_are(T, K):
    """parts of a contraction are written and read in whole groups of 64, so that up to 64 outputs cost the same"""
    size = load_library().qb_linear_fwd_workspace_nbytes
    for codes in (False, True):
        assert len({size(linear(T, N, K, codes)) for N in (1, 2, 16, 33, 63, 64)}) == 1


def plan_forward(T, N, K, codes):
    rule, parts = ctypes.CDLL(LIB_PATH)._ZN2qb15linear_fwd_planEPK9qb_linearPi, ctypes.c_int()
    size = rule(linear(T, N, K, codes), ctypes.byref(parts))
    return size, parts.value


def plan_backward(T, N, K, dX, dW):
    rule, x, w = ctypes.CDLL(LIB_PATH)._ZN2qb15linear_bwd_planEPK15qb_linear_gradsPiS3_, ctypes.c_int(), ctypes.c_int()
    size = rule(ctypes.byref(LinearGrads(type=0, act=0, T=T, N=N, K=K, dY=P, dy_row=N, W=P, X=P, x_row=K, dX=P if dX else None, dW=P if dW else None)), ctypes.byref(x), ctypes.byref(w))
    return size, x.value, w.value


def test_forward_calls_on_the_gpu_take_every_kernel():
    """what test_gpu_linear_plans.py runs, by the plan that it gets: another rule would have to bring other calls"""
    few, tiles, streams = set(), set(), set()
    for T, N, K in FORWARD:
        for codes in (False, True):
            size, parts = plan_forward(T, N, K, codes)
            if size < 0:
                units = -(-K // (512 * parts))
                tokens = 16 if T <= 16 else 32 if T <= 32 else 64
                few.add((-size, tokens, parts > 1, 0 if size < -1 else 1 if units == 1 else 4 if units > 2 and tokens < 64 else 2))
            else:
                tiles.add((size, parts > 1))
                streams.add((size, N % 64 == 0))
    assert few >= {(1, t, cut, u) for t in (16, 32) for cut in (False, True) for u in (1, 2, 4)} | {(1, 64, False, 1), (1, 64, False, 2)}
    assert few >= {(2, t, cut, 0) for t in (16, 32) for cut in (False, True)} | {(2, 64, False, 0)}
    assert tiles >= {(s, cut) for s in (0, 1, 2) for cut in (False, True)} | {(3, False), (4, False)}
    assert streams >= {(s, whole) for s in (3, 4) for whole in (False, True)}


def test_backward_calls_on_the_gpu_take_every_kernel():
    got = set()
    for shape in BACKWARD:
        for dX, dW, _ in NEEDS:
            size, x, w = plan_backward(*shape, dX, dW)
            got.add((size, dX, dW, x > 1, w > 1))
    for size in range(4):  # least .. large: both gradients, one alone; nothing, either one or both cut into parts
        want = {(size, True, True, x, w) for x in (False, True) for w in (False, True)} | {(size, True, False, x, False) for x in (False, True)} | {
            (size, False, True, False, w) for w in (False, True)}
        assert got >= want, want - got


def test_no_plan_cuts_the_large_tiles_of_the_forward():
    """their kernel has no parts"""
    for T in (65, 300, 3000, 30000):
        for N in (64, 1000, 9000):
            for K in (64, 1024, 32768):
                size, parts = plan_forward(T, N, K, False)
                assert size < 3 or parts == 1


FORWARD_TILES = {0: (64, 64, 256), 1: (64, 128, 256), 2: (128, 128, 256), 3: (128, 256, 512), 4: (256, 256, 512)}  # outputs, tokens, threads
BACKWARD_TILES = {0: (64, 64, 256), 1: (64, 128, 256), 2: (128, 128, 256), 3: (256, 256, 512)}                     # inputs, tokens or neurons, threads
MEMORY = 300e9  # bytes: a result beyond it has nowhere to lie


def test_no_launch_has_2_to_32_threads():
    """more of them are not refused, some just do not run: tiles and joins of every size of call that memory has room for"""
    for t in range(7, 25):
        for n in range(21):
            T, N = 1 << t, 1 << n
            if T * N * 2 > MEMORY:
                continue
            for K in (64, 1024, 32768):
                size, parts = plan_forward(T, N, K, False)
                outputs, tokens, threads = FORWARD_TILES[size]
                assert -(-N // outputs) * -(-T // tokens) * parts * threads < 1 << 32
                assert parts == 1 or T * -(-N // 64) * 16 < 1 << 32
                for dX, dW in ((True, True), (True, False), (False, True)):
                    if T * K * 2 * dX > MEMORY or N * K * 2 * dW > MEMORY:
                        continue
                    size, x, w = plan_backward(T, N, K, dX, dW)
                    inputs, rows, threads = BACKWARD_TILES[size]
                    assert -(-K // inputs) * (-(-T // rows) * x * dX + -(-N // rows) * w * dW) * threads < 1 << 32
                    assert (T * (x > 1) + N * (w > 1)) * K // 4 < 1 << 32
