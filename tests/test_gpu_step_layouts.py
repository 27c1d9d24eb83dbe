"""Decode behind shared prefixes: where the partials lie (by request, or by range with room for the largest group), one workspace for steps of all sizes, and lists and prefixes
that are longer than stated."""
import numpy as np
import pytest
import torch

from esp_checks import check_o_lse
from paper_2404_09526_amd import binding as esp
from test_gpu_step import f64, form, poisoned, shared_inputs, shared_reference, shared_workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def checked(call, both, cuda, what, **kw):
    Or, Lr = shared_reference(call, both, cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, **kw)
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), what)
    return O, LSE


UNEQUAL = [
    ("one-large", [200] + [1] * 40, [500] * 41, [3, 0, 40] * 80, 8, 2), ("one-large-last", [1] * 70 + [90], [130] * 71, [9] * 160, 16, 16),
    ("one-long", [3] * 20, [4500] + [40] * 19, [5, 70, 0] * 20, 8, 2), ("one-long-last", [1, 2] * 33, [33] * 65 + [9001], [7] * 99, 4, 1),
    ("both", [1] * 30 + [66] + [2] * 30, [64] * 30 + [2100] + [0, 700] * 15, [20, 0, 3, 1, 64, 65] * 26, 32, 8),
]


@pytest.mark.parametrize("name,groups,prefixes,lens,Hq,Hkv", UNEQUAL, ids=[u[0] for u in UNEQUAL])
def test_unequal_groups(cuda, form, name, groups, prefixes, lens, Hq, Hkv):  # noqa: F811
    call, both = shared_inputs(cuda, groups, prefixes, lens[:sum(groups)], Hq, Hkv, 81)
    O, LSE = checked(call, both, cuda, name, workspace=shared_workspace(call, cuda))
    # a larger block changes nothing
    big = poisoned(300 << 20, cuda)
    O2, L2 = esp.esp_partial_attn_decode_shared(**call, workspace=big)
    assert torch.equal(O, O2) and torch.equal(LSE, L2)


def test_one_workspace_for_all_steps(cuda, form):  # noqa: F811
    """A block for the largest step takes every smaller one; nothing is written behind what the call asks for."""
    steps = [([64], [2051], [1600] * 64), ([64], [2051], [50] * 64), ([64], [2051], [100] * 64), ([30, 20], [2000, 51], [7] * 50), ([64], [2051], [0] * 64), ([3], [2051], [1600, 1, 0]),
             ([64], [0], [100] * 64), ([1], [1], [1])]
    ws = poisoned(esp.esp_decode_shared_workspace_bytes(64, 2, 2051, 2051, 64, 102400, 1600, 32, 8, 128), cuda)
    for i, (groups, prefixes, lens) in enumerate(steps):
        call, both = shared_inputs(cuda, groups, prefixes, lens, 32, 8, 82 + i)
        ws.fill_(0xFF)
        checked(call, both, cuda, str(i), workspace=ws)
        asked = shared_workspace(call, cuda).numel()
        assert asked <= ws.numel() and (ws[asked:] == 0xFF).all(), i


@pytest.mark.parametrize("groups", [[2, 90], [3] * 40], ids=["two", "many"])
def test_a_prefix_longer_than_stated_is_read_as_far_as_that(cuda, form, groups):  # noqa: F811
    prefixes = [3000] + [700, 65] * 20
    call, both = shared_inputs(cuda, groups, prefixes[:len(groups)], [5, 0, 40] * 40 if len(groups) > 2 else [6] * 92, 8, 2, 83)
    call["max_prefix"] = 645                                            # past a tile, within a range
    b = 0
    for g, n in enumerate(groups):
        for _ in range(n):
            both[b] = np.concatenate([both[b][:min(prefixes[g], 645)], both[b][prefixes[g]:]])
            b += 1
    checked(call, both, cuda, "cut", workspace=shared_workspace(call, cuda))
    call["max_prefix"] = 0
    for b, g in enumerate(np.repeat(np.arange(len(groups)), groups)):
        both[b] = both[b][min(prefixes[g], 645):]
    checked(call, both, cuda, "none")


@pytest.mark.parametrize("groups,prefixes,lens", [([4], [300], [40, 0, 1, 77]), ([40, 3], [700, 64], [9] * 43), ([200], [3000], [0, 5] * 100)])
def test_slots_past_the_offsets_belong_to_no_request(cuda, form, groups, prefixes, lens):  # noqa: F811
    """Lists with spare room, as lists made on the GPU have: what lies behind the last offset is never attended."""
    call, both = shared_inputs(cuda, groups, prefixes, lens, 8, 2, 84)
    spare = torch.arange(5000, dtype=torch.int32, device=cuda) % call["k_pool"].shape[0]
    for name in ("prefix_slots", "slot_idx"):
        call[name] = torch.cat([call[name], spare])
    checked(call, both, cuda, "spare room", workspace=shared_workspace(call, cuda))


@pytest.mark.parametrize("past", [3, 700])
@pytest.mark.parametrize("groups,prefixes,lens", [([4], [300], [40, 0, 1, 77]), ([40, 3], [700, 64], [9] * 42 + [300]), ([200], [3000], [0, 5] * 99 + [5, 0])])
def test_offsets_past_the_slots_read_none(cuda, form, groups, prefixes, lens, past):  # noqa: F811
    """Offsets that end behind the lists, within the last range and ranges further: what is there counts, in every range of every request, and no more."""
    call, both = shared_inputs(cuda, groups, prefixes, lens, 8, 2, 85)
    free = np.setdiff1d(np.arange(call["k_pool"].shape[0]), np.concatenate(both))
    bad = torch.full((5000,), int(free[0]), dtype=torch.int32, device=cuda)   # (behind the lists in memory: a row of the pool that is NaN)
    for slots, offs in (("prefix_slots", "prefix_offsets"), ("slot_idx", "seq_offsets")):
        n = call[slots].numel()
        call[slots] = torch.cat([call[slots], bad])[:n]
        call[offs] = call[offs].clone()
        call[offs][-1] += past
    checked(call, both, cuda, "past the end", workspace=shared_workspace(call, cuda))
    call["max_prefix"], call["max_len"] = call["prefix_slots"].numel(), call["slot_idx"].numel()
    checked(call, both, cuda, "past the end", workspace=shared_workspace(call, cuda))
