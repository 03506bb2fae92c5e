"""The attention backward's rules for its workspace, as host functions of the library."""
import ctypes
import itertools

from paper_1909_05840_amd.binding import LIB_PATH


def test_parts_of_keys_never_pass_the_room_for_them():
    """A tile of keys writes its sums in as many parts as its sequence's own length asks for, which the device reads; the host reserves by the
    longest length that the caller names.  A sequence that is longer than that has undefined results, but writes no part beyond the room."""
    rule = ctypes.CDLL(LIB_PATH)._ZN2qb19attention_row_partsEllllbiiiiPi
    i64, reserved = ctypes.c_int64, ctypes.c_int()
    rule.restype, rule.argtypes = ctypes.c_int, [i64] * 4 + [ctypes.c_bool] + [ctypes.c_int] * 4 + [ctypes.POINTER(ctypes.c_int)]
    several = 0
    for pairs, group, max_q, causal, dim in itertools.product((1, 12, 96, 384), (1, 3, 4, 80), (0, 1, 64, 500, 4000), (False, True), (64, 128)):
        for max_k, nq, nk in itertools.product((128, 500, 8192), (0, 1, 63, 500, 700, 4001, 70000), (1, 500, 9000)):
            for first_key in range(0, nk, 2048):
                parts = rule(pairs, group, max_q, max_k, causal, dim, nq, nk, first_key, reserved)
                assert 1 <= parts <= reserved.value, (pairs, group, max_q, max_k, causal, dim, nq, nk, first_key)
                several += parts > 1
    assert several > 1000
