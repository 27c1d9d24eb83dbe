"""Sizes and scales at which the calls on the pool in 4 bits, of attention weights and of eviction answer on the host."""
import random

import pytest

from test_q4_checks import F, P, lib, nul, one  # noqa: F401


@pytest.mark.parametrize("scale", [2.36e38, 2.5e38, 3e38, 3.4e38])
def test_a_scale_whose_factor_is_infinite_is_refused(lib, scale):  # noqa: F811
    """Exponentials are taken to the base 2: the scale times log2(e) has to be a number too (a score of 0 would be NaN)."""
    need = lib.esp_decode_q4_workspace_bytes(3, 100, 60, 32, 8, 128)
    # (a workspace that is too small, no requests: refused, or done, before anything is launched)
    decode = lambda s: lib.lib.esp_partial_attn_decode_q4(one, one, one, 544, 128, one, one, 3, 100, 60, 32, 8, 128, F(s), one, one, one, need - 1, nul)  # noqa: E731
    assert decode(scale) == lib.ESP_ERR_INVALID_ARG and "softmax_scale" in lib.last_error()
    assert decode(2.35e38) == lib.ESP_ERR_WORKSPACE
    tail = lambda s: (128, one, one, 0, 0, 0, nul, 0, 0, nul, nul, 32, 8, 128, F(s), F(0.9), 1, one, nul)  # noqa: E731
    for call in (lambda s: lib.lib.esp_accumulate_attn_weights(one, one, one, *tail(s)), lambda s: lib.lib.esp_accumulate_attn_weights_q4(one, one, one, 544, *tail(s))):
        assert call(scale) == lib.ESP_ERR_INVALID_ARG and "softmax_scale" in lib.last_error()
        assert call(2.35e38) == lib.ESP_OK


def test_the_workspace_of_decode_rises_with_every_size(lib):  # noqa: F811
    """One that is large enough for a call is so for any with as many requests, entries and heads, or fewer."""
    rng = random.Random(1)
    kv = [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 16, 17, 20, 24, 25, 32, 36, 40]
    for _ in range(4000):
        B, T, G, H = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 24)), rng.randint(1, 40), rng.choice(kv)
        b, t, h = rng.choice([B, rng.randint(0, B)]), rng.choice([T, rng.randint(0, T)]), rng.choice([x for x in kv if x <= H])
        hq = rng.randint(1, G * H // h) * h
        assert lib.esp_decode_q4_workspace_bytes(B, T, T, G * H, H, 128) >= lib.esp_decode_q4_workspace_bytes(b, t, t, hq, h, 128) > 0, (B, T, G, H, b, t, hq, h)


def test_lists_without_room_overlap_nothing(lib):  # noqa: F811
    """A capacity of 0, or no entries, with a pointer into another array."""
    need = lib.esp_evict_workspace_bytes(3, 100, 60)
    at = {n: P(1 << (20 + i)) for i, n in enumerate(("sums", "idx", "pos", "off", "ko", "ks", "kp", "fo", "fs", "ws"))}

    def call(S=128, total=100, max_len=60, kc=100, fc=100, **other):
        a = dict(at, **other)                                         # (a workspace that is too small: refused last, nothing is launched)
        return lib.lib.esp_evict_slots(a["sums"], S, a["idx"], a["pos"], a["off"], 3, total, max_len, nul, 5, 1, 1, kc, a["ko"], a["ks"], a["kp"], fc, a["fo"], a["fs"], a["ws"],
                                       need - 1 if total else 1, nul)
    inside = P((1 << 25) + 200)                                       # of kept_slots
    for kw in (dict(), dict(fc=0, fs=inside), dict(kc=0, ks=P((1 << 28) + 40), kp=P((1 << 28) + 40)), dict(S=0, sums=inside), dict(total=0, max_len=0, idx=inside, pos=inside)):
        assert call(**kw) == lib.ESP_ERR_WORKSPACE, kw
    for kw in (dict(fs=inside), dict(fc=1, fs=inside), dict(S=1, sums=inside), dict(idx=inside), dict(pos=inside)):
        assert call(**kw) == lib.ESP_ERR_INVALID_ARG and "overlap" in lib.last_error(), kw
