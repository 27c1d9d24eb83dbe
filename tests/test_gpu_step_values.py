"""Decode behind shared prefixes with infinities among the values: they show as themselves in the elements that see them, also in the last row of a list, which tiles
that are not full repeat with weight 0."""
import pytest
import torch

from paper_2404_09526_amd import binding as esp
from test_gpu_step import form, shared_inputs, shared_workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,prefixes,Hq", [(2, [300, 310], 2), (30, [301, 33], 2), (60, [65, 1001], 2), (125, [513, 300], 2), (100, [9000, 4001], 8), (68, [20001, 19999], 16)])
def test_infinite_values_show_as_themselves(cuda, form, n, prefixes, Hq):  # noqa: F811
    """The last row of a prefix, the last of a request's own, and one in the middle; every other element keeps its bits."""
    call, _ = shared_inputs(cuda, [n, n], prefixes, [3, 35] * n, Hq, 2, 71)
    ws, G, inf = shared_workspace(call, cuda), Hq // 2, float("inf")
    own = call["slot_idx"].long()
    v = call["v_pool"]
    rows = [(call["prefix_slots"][prefixes[0] - 1].long(), 1, 5, inf, slice(0, n)), (call["prefix_slots"][-1].long(), 0, 127, -inf, slice(n, 2 * n)),
            (call["prefix_slots"][17].long(), 0, 64, -inf, slice(0, n)), (own[2], 1, 9, -inf, slice(0, 1)), (own[37], 0, 31, inf, slice(1, 2)), (own[-1], 1, 0, inf, slice(2 * n - 1, 2 * n))]
    for at, h, d, _, _ in rows:
        v[at, h, d] = 0
    O0, L0 = esp.esp_partial_attn_decode_shared(**call, workspace=ws)
    assert torch.isfinite(O0).all()
    for at, h, d, x, _ in rows:
        v[at, h, d] = x
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=ws)
    want = O0.clone()
    for _, h, d, x, who in rows:
        want[who, h * G:(h + 1) * G, d] = x
    assert torch.equal(O, want) and torch.equal(LSE, L0)
