"""The 16-bit linears' rules for tiles and for parts of their contractions, on the host (no GPU needed)."""
import ctypes

import pytest

from paper_1909_05840_amd.binding import LinearGrads, LinearLayer, load_library

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
