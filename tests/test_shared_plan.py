"""Which calls behind shared prefixes run in one launch, and on workgroups of how many wavefronts, without a GPU: that the rule answers for itself, and that a test may set
it for its own thread."""
import threading

import pytest

from paper_2404_09526_amd import binding as esp

BIG = 2**31 - 1


def plan(groups, prefixes, lens, Hq, Hkv):
    return esp.esp_debug_decode_shared_plan(sum(groups), len(groups), sum(prefixes), max(prefixes), max(groups), sum(lens), max(lens), Hq, Hkv)


def test_what_the_estimates_say():
    assert plan([4], [300], [40] * 4, 4, 4) == 2                         # few short requests
    assert plan([64], [2051], [750] * 64, 32, 8) == 4 and plan([16], [65536], [300] * 16, 32, 32) == 4
    assert plan([136], [20000], [7] * 136, 16, 16) == 8                  # a long prefix and little else
    assert plan([3, 2], [0, 0], [50, 0, 7, 1, 1], 8, 2) == esp.esp_debug_decode_plan(5, 59, 50, 8, 2)   # no prefix: plain decode


@pytest.mark.parametrize("sizes", [(-1, 1, 9, 9, 0, 5, 5, 8, 2), (3, 1, 9, 10, 3, 5, 5, 8, 2), (3, 1, 9, 9, 4, 5, 5, 8, 2), (3, 0, 9, 9, 3, 5, 5, 8, 2), (3, 1, 9, 9, 3, 5, 6, 8, 2), (3, 1, 9, 9, 3, 5, -1, 8, 2),
                                   (3, 1, 9, 9, 3, 5, 5, 8, 3)])
def test_sizes_that_are_not_valid(sizes):
    assert esp.esp_debug_decode_shared_plan(*sizes) == 0


def test_a_plan_is_set_for_the_thread_that_asks():
    sizes = (64, 1, 2051, 2051, 64, 48000, 4096, 32, 8)
    for n in (2, 4, 8):
        assert esp.esp_debug_set_decode_plan(n) == 0
        try:
            there = []
            t = threading.Thread(target=lambda: there.append(esp.esp_debug_decode_shared_plan(*sizes)))
            t.start()
            t.join()
            assert esp.esp_debug_decode_shared_plan(*sizes) == n and there == [4]
            assert esp.esp_debug_decode_plan(4, 1283, 485, 4, 4) == (2 if n == 2 else 1)
            # a request's keys in one launch are counted in 32 bits: lists that may be longer are ranges, whatever is asked for
            assert esp.esp_debug_decode_shared_plan(1, 1, BIG, BIG, 1, BIG, BIG, 8, 2) in (4, 8)
            assert esp.esp_debug_decode_shared_plan(1, 1, BIG, BIG, 1, 1, 1, 8, 2) in (4, 8)
            assert esp.esp_debug_decode_shared_plan(1, 1, BIG, BIG, 1, 1, 0, 8, 2) == n
        finally:
            assert esp.esp_debug_set_decode_plan(0) == n
    for other in (3, 5, 7, 16, -4):
        assert esp.esp_debug_set_decode_plan(other) == 0 and esp.esp_debug_set_decode_plan(0) == 0
