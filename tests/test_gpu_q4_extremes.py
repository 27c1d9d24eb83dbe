"""Decode over the pool in 4 bits at the ends of what its bytes can say: an infinite value in the last row of a list, and rows as large and as small as they are kept.

A weight is off by half a unit of bf16 (2^-8 of it) in the products and in the sum they are divided by, the result by half a unit once it is rounded; fp32 sums of up to 2^12 terms and
the exponentials are within 2^-11.  That is 2^-7 + 2^-11 of the sum of weights times magnitudes, and 2^-8 of the result."""
import numpy as np
import pytest
import torch

import oracle
import q4_reference as q4
from esp_checks import check_o_lse
from paper_2404_09526_amd import binding as esp
from test_gpu_q4 import decode_case, from_bits, i32, offsets, pools

pytestmark = pytest.mark.gpu

INFINITE = 254                                                        # the scale 2^127: a code of 2 and more is no finite bf16 number


@pytest.mark.parametrize("lens", [[1], [33, 2], [600, 31, 5], [1600, 64, 17], [5000, 1, 0, 100], [65] * 300], ids=lambda x: f"{len(x)}x{max(x)}")
@pytest.mark.parametrize("hq,hkv,layout", [(8, 8, "apart"), (32, 8, "joint"), (4, 4, "joint"), (160, 8, "joint"), (80, 4, "apart"), (12, 12, "joint"), (6, 3, "joint"), (2, 2, "apart"),
                                           (4, 1, "joint"), (32, 1, "joint"), (20, 1, "apart")])
def test_an_infinite_value_in_the_last_row_shows_as_itself(cuda, hq, hkv, layout, lens):
    """What a list's tokens leave of a tile is the last one's slot again, with no weight: 0 times an infinity must not come of it.  (Append writes no such rows; the format has them.)"""
    c = decode_case(cuda, lens, hq, hkv, layout, hq + len(lens))
    some = [b for b, n in enumerate(lens) if n]
    rows = c["args"][2].cpu().numpy().copy()
    head, element, sign = np.arange(hkv), 7 * np.arange(hkv) % 128, np.where(np.arange(hkv) % 2, -1.0, 1.0)
    finite = q4.bf16_values(c["v"])
    for b in some:
        s = c["slot"][c["off"][b + 1] - 1]
        for h in head:
            block, at = element[h] // 32, element[h] // 2
            rows[s, h, 16 * block:16 * block + 16] = 0
            rows[s, h, at] = (0x4 if sign[h] > 0 else 0xC) << 4 * (element[h] % 2)
            rows[s, h, 64 + block] = INFINITE
            finite[s, h, 32 * block:32 * block + 32] = 0
    c["args"][2].copy_(torch.from_numpy(rows).to(cuda))
    O, LSE = esp.esp_partial_attn_decode_q4(*c["args"])
    O = O.double().cpu().numpy()
    Or, Lr = oracle.partial_attn_decode_all(c["q"], c["k"], q4.bf16_bits(finite), c["slot"], c["off"], 128 ** -0.5)
    G = hq // hkv
    for h in head:
        mine = np.s_[some, h * G:(h + 1) * G, element[h]]
        assert (O[mine] == sign[h] * np.inf).all(), (h, O[mine])
        O[mine] = Or[mine] = 0
    check_o_lse(O.reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), f"{hq}/{hkv} {layout}")


def lone_case(dev, n, hq, hkv, layout, at, score, codes_v, scale_v, others):
    """One request of n keys of score 0 and one, at `at`, of score `score`; V's rows there are codes_v with scale_v everywhere, `others` with 127 elsewhere."""
    rows_k, rows_v = np.zeros((n, hkv, 68), np.uint8), np.full((n, hkv, 68), others, np.uint8)
    rows_k[..., 64:] = rows_v[..., 64:] = 127
    rows_k[at, :, 0] = 0x2                                            # element 0: 1
    rows_v[at, :, :64], rows_v[at, :, 64:] = codes_v, scale_v
    slot = np.random.default_rng(n).permutation(n)
    kp, vp = pools(dev, n, hkv, layout)
    for pool, rows in ((kp, rows_k), (vp, rows_v)):
        placed = np.empty_like(rows)
        placed[slot] = rows
        pool.copy_(torch.from_numpy(placed).to(dev))
    q = np.zeros((1, hq, 128))
    q[..., 0] = score
    return (from_bits(q4.bf16_bits(q), dev), kp, vp, i32(slot, dev), i32([0, n], dev), n), q4.values(rows_k), q4.values(rows_v), q


def check_lone(args, k, v, q, what):
    O, LSE = esp.esp_partial_attn_decode_q4(*args, softmax_scale=1.0)
    O, LSE = O.double().cpu().numpy()[0], LSE.double().cpu().numpy()[0]
    G = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        s = k[:, h // G] @ q[0, h]
        p = np.exp(s - s.max())
        want, size = p @ v[:, h // G] / p.sum(), p @ np.abs(v[:, h // G]) / p.sum()
        off = np.abs(O[h] - want)
        assert (off <= (2.0 ** -7 + 2.0 ** -11) * size + 2.0 ** -8 * np.abs(want)).all(), (what, h, O[h][:4], want[:4])
        assert abs(LSE[h] - (s.max() + np.log(p.sum()))) <= 1e-4 * max(1.0, abs(s.max())), what


LONE_HEADS = [(8, 8, "apart"), (32, 8, "joint"), (4, 4, "joint"), (160, 8, "joint"), (6, 3, "joint"), (4, 1, "joint"), (32, 1, "apart")]


@pytest.mark.parametrize("score", [0.0, 3.0, 6.90625, 7.5, 30.0])
@pytest.mark.parametrize("hq,hkv,layout", LONE_HEADS)
def test_the_largest_rows_after_others_that_weigh_less(cuda, hq, hkv, layout, score):
    """A row of the largest values that are stored, 6 * 2^125, 2^10 times as heavy as those before it: the mean is a finite number, and so is all on the way to it."""
    for n, at in ((600, 599), (600, 300), (3000, 2900)):
        check_lone(*lone_case(cuda, n, hq, hkv, layout, at, score, 0xF7, 252, 0x22), f"{n} {at}")


@pytest.mark.parametrize("score", [0.0, 6.90625, 30.0])
@pytest.mark.parametrize("hq,hkv,layout", LONE_HEADS)
def test_the_smallest_rows(cuda, hq, hkv, layout, score):
    """The smallest values that are stored, 0.5 * 2^-125, alone, beside zeros and beside each other."""
    for n, at in ((1, 0), (600, 599), (3000, 100)):
        case = lone_case(cuda, n, hq, hkv, layout, at, score, 0x91, 2, 0)
        if score == 0:                                                # all rows alike
            case[0][2][..., :64], case[0][2][..., 64:] = 0x91, 2
            case[2][:] = case[2][at]
        elif score < 30 and n > 1:
            continue                                                  # (a part of the smallest bf16 number: it has fewer bits)
        check_lone(*case, f"{n} {at}")
