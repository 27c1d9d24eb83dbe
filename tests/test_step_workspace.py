"""What decode behind shared prefixes asks for as a workspace: it rises with every size, so that a program may size its block once, for the largest step that it expects, and
it stays near what the partials of long ranges need, however unequal the groups are."""
import ctypes
import math
import random

import pytest

from paper_2404_09526_amd import binding as esp

HEADS = [(4, 4), (8, 8), (16, 16), (32, 32), (64, 64), (8, 4), (16, 8), (8, 2), (32, 8), (32, 1), (24, 3), (64, 8), (66, 2)]


def need(B, n_groups, prefix_total, max_prefix, max_group, total, Hq, Hkv):
    return esp.esp_decode_shared_workspace_bytes(B, n_groups, prefix_total, max_prefix, max_group, total, total, Hq, Hkv, 128)


def drawn(rng):
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))  # noqa: E731
    B, P = log(1, 4000), log(1, 3000000)
    return B, log(1, 300), P, rng.randint(1, P), rng.randint(0, B), rng.choice([0, log(1, 5000000)])


@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_it_rises_with_every_size(Hq, Hkv):
    rng = random.Random(Hq * 100 + Hkv)
    for _ in range(4000):
        sizes = drawn(rng)
        less = [rng.choice([x, x, rng.randint(lo, x), max(lo, x - 1)]) for x, lo in zip(sizes, (1, 1, 0, 0, 0, 0))]
        less[3], less[4] = min(less[3], less[2]), min(less[4], less[0])
        assert 0 < need(*less, Hq, Hkv) <= need(*sizes, Hq, Hkv), (less, sizes)


def test_the_steps_of_one_batch():
    """64 requests behind 2051 tokens whose own lists grow."""
    sizes = [need(64, 1, 2051, 2051, 64, 64 * n, 32, 8) for n in (0, 1, 50, 100, 200, 800, 1600, 5000, 20000)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 8), (64, 8)])
def test_it_covers_plain_decode_and_is_refused_one_byte_short(Hq, Hkv):
    rng, one = random.Random(5), ctypes.c_void_p(256)                   # never dereferenced
    for i in range(300):
        B, n, P, mp, mg, T = drawn(rng)
        if i % 3 == 0:
            P = mp = mg = 0                                             # no prefix: that call is plain decode
        n_bytes = need(B, n, P, mp, mg, T, Hq, Hkv)
        assert n_bytes >= esp.esp_decode_workspace_bytes(B, T, T, Hq, Hkv, 128)
        status = esp.lib.esp_partial_attn_decode_shared(one, one, one, 1 << 24, one, one, one, n, P, mp, mg, one, one, B, T, T, Hq, Hkv, 128, ctypes.c_float(0.1), one, one, one,
                                                        n_bytes - 1, ctypes.c_void_p(0))
        assert status == esp.ESP_ERR_WORKSPACE


@pytest.mark.parametrize("B,n_groups,prefix,max_group,own", [(256, 16, 20000, 200, 600), (320, 65, 30000, 256, 300), (1024, 513, 16000, 512, 500), (4000, 2000, 4096, 3000, 50)])
def test_unequal_groups_do_not_take_the_largests_room_each(B, n_groups, prefix, max_group, own):
    """A row for each range of 4096 keys of each request, or 128 MiB, and the same of the own lists."""
    Hq, row = 32, 32 * 520
    most = max(128 << 20, B * -(-prefix // 4096) * row) + max(128 << 20, (B * own // 512 + B) * row) + 512
    assert need(B, n_groups, n_groups * prefix, prefix, max_group, B * own, Hq, 8) <= most
    # and few requests behind one of many long prefixes take no more than the prefixes have ranges, for the largest group
    slots = (n_groups * prefix // 4096 + n_groups) * 2 * row
    assert need(2 * n_groups, n_groups, n_groups * prefix, n_groups * prefix, 2, 0, Hq, 8) <= max(128 << 20, slots) + 256


def test_sizes_past_64_bits_are_refused_and_not_wrapped():
    one, big = ctypes.c_void_p(256), 2**31 - 1
    for sizes in ((big // 64, big, big, big, big // 64, big), (big // 64, 1, big, big, big // 64, 0)):
        n = need(*sizes, 64, 8)
        assert n >= 1 << 50
        B, g, P, mp, mg, T = sizes
        status = esp.lib.esp_partial_attn_decode_shared(one, one, one, 1 << 24, one, one, one, g, P, mp, mg, one, one, B, T, T, 64, 8, 128, ctypes.c_float(0.1), one, one, one, 1 << 45,
                                                        ctypes.c_void_p(0))
        assert status == esp.ESP_ERR_WORKSPACE
