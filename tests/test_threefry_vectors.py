"""Dropout's generator, as the tests and the plain operators write it down, against the published test vectors of Threefry-2x32 with 13 rounds
(the authors' library of the paper, SC 2011: counter, key, result)."""
import pytest
import torch

from perf import operators
from test_gpu_attention import draws as draws_of_weights

VECTORS = [((0x00000000, 0x00000000), (0x00000000, 0x00000000), (0x9D1C5EC6, 0x8BD50731)),
           ((0xFFFFFFFF, 0xFFFFFFFF), (0xFFFFFFFF, 0xFFFFFFFF), (0xFD36D048, 0x2D17272C)),
           ((0x243F6A88, 0x85A308D3), (0x13198A2E, 0x03707344), (0xBA3E4725, 0xF27D669E))]


def int64(low, high):
    v = low | high << 32
    return v - (1 << 64) if v >> 63 else v


@pytest.mark.parametrize("counter,key,want", VECTORS)
def test_published_vectors(counter, key, want):
    seed = int64(*key)
    words = operators._threefry(torch.tensor([counter[0]]), torch.tensor([counter[1]]), torch.tensor([seed]))
    assert [int(w) for w in words] == list(want)
    halves = [h for w in want for h in (w & 0xFFFF, w >> 16)]
    low32 = lambda v: torch.tensor([v - (1 << 32) if v >> 31 else v], dtype=torch.int32)  # noqa: E731
    assert operators._draws(low32(counter[0]), low32(counter[1]), torch.tensor([seed])).reshape(-1).tolist() == halves
    index = torch.arange(4)
    assert draws_of_weights(torch.tensor([counter[0]]), torch.tensor([counter[1]]), index, seed).tolist() == halves


@pytest.mark.gpu
def test_the_kernels_draws_are_the_published_ones(qb):
    """with key 0 the first four values take the draws of counter 0: each is kept at a threshold of its draw, and dropped one above"""
    x, seed = torch.ones(4, device="cuda:0"), torch.zeros(1, dtype=torch.int64, device="cuda:0")
    for i, draw in enumerate((0x5EC6, 0x9D1C, 0x0731, 0x8BD5)):
        print("value", i, "draw", draw, flush=True)
        assert qb.qb_dropout_fwd(x, draw / 65536, seed)[i] != 0
        assert qb.qb_dropout_fwd(x, (draw + 1) / 65536, seed)[i] == 0
