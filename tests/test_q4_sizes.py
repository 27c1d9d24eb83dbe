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
