"""softmax_scale = 0: every visible key weighs the same, and what hides the others must not depend on the scale.  O is the mean of the visible
rows, LSE the logarithm of their number, in every call and form."""
import numpy as np
import pytest
import torch

import oracle
from esp_checks import check_o_lse
from paper_2404_09526_amd import binding as esp
from paper_2404_09526_amd import workloads as wl
from test_gpu_step import f64, shared_inputs, shared_workspace

pytestmark = pytest.mark.gpu


def means(call, both):
    """The definition: mean of the rows, logarithm of their number; 0 and -inf where there are none."""
    v, Hq = f64(call["v_pool"]), call["q"].shape[1]
    G = Hq // v.shape[1]
    O = np.stack([np.repeat(v[rows].mean(0), G, 0) if len(rows) else np.zeros((Hq, 128)) for rows in both])
    with np.errstate(divide="ignore"):
        return O, np.repeat(np.log(np.array([len(rows) for rows in both], float))[:, None], Hq, 1)


@pytest.mark.parametrize("plan", [0, 1, 2], ids=["by-estimate", "ranges", "one-launch"])
@pytest.mark.parametrize("groups,prefixes,lens,Hq,Hkv", [([5], [517], [3, 64, 31, 0, 130], 32, 8), ([3], [0], [50, 0, 7], 8, 2), ([2, 20, 1], [65, 330, 0], [9, 33, 0] + [5] * 20, 16, 4),
                                                         ([40], [1031], [1] * 40, 32, 8), ([136], [20000], [7] * 136, 16, 16)],
                         ids=["one-tile", "no-prefix", "two-tiles", "blocks", "long"])
def test_shared_decode(cuda, plan, groups, prefixes, lens, Hq, Hkv):
    call, both = shared_inputs(cuda, groups, prefixes, lens, Hq, Hkv, 61)
    before = esp.esp_debug_set_decode_plan(plan)
    try:
        O, LSE = esp.esp_partial_attn_decode_shared(**call, softmax_scale=0.0, workspace=shared_workspace(call, cuda))
    finally:
        esp.esp_debug_set_decode_plan(before)
    Or, Lr = means(call, both)
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "shared")


@pytest.mark.parametrize("plan", [1, 2], ids=["ranges", "one-launch"])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (16, 8), (32, 8), (66, 2), (6, 3)])
def test_decode(cuda, plan, Hq, Hkv):
    lens = [1, 40, 0, 700, 33, 64]
    dc = wl.decode_pool(f"scale-0 ({Hq}/{Hkv})", lens, 4096, Hq, Hkv, 62, cuda, n_new=0)
    off, slots = wl.host_i32(dc.seq_offsets), wl.host_i32(dc.slot_idx)
    before = esp.esp_debug_set_decode_plan(plan)
    try:
        O, LSE = esp.esp_partial_attn_decode(dc.q, dc.k_pool, dc.v_pool, dc.slot_idx, dc.seq_offsets, max(lens), softmax_scale=0.0)
    finally:
        esp.esp_debug_set_decode_plan(before)
    Or, Lr = means(dict(q=dc.q, v_pool=dc.v_pool), [slots[off[b]:off[b + 1]] for b in range(len(lens))])
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), dc.name)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Tq,Tkv,Hq,Hkv", [(40, 70, 8, 2), (300, 1000, 4, 4), (1, 33, 8, 8), (130, 130, 8, 2)])
def test_prefill(cuda, each_prefill_plan, Tq, Tkv, Hq, Hkv, causal):
    pc = wl.contiguous_prefill("scale-0", Tq, Tkv - Tq, [(0, Tkv)], Hq, Hkv, 63, cuda)
    s = pc.shards[0]
    O, LSE = esp.esp_partial_attn_prefill(pc.q, s.k, s.v, pc.q_pos, s.kv_pos, softmax_scale=0.0, causal=causal)
    Or, Lr = oracle.partial_attn_all(wl.bits(pc.q), wl.bits(s.k), wl.bits(s.v), wl.host_i32(pc.q_pos), wl.host_i32(s.kv_pos), 0.0, causal)
    n = np.where(causal, Tkv - Tq + 1 + np.arange(Tq), Tkv)
    assert np.allclose(Lr, np.log(n)[:, None])                        # the oracle hides by position, whatever the scale
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "prefill")
