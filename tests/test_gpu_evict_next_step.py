"""The step after an eviction: the kept lists are rows of a block table with pages of one token, the freed slots its free pages."""
import numpy as np
import pytest
import torch

import oracle
import q4_reference as q4
from esp_checks import check_o_lse
from paper_2404_09526_amd import binding as esp
from test_gpu_q4 import decode_case, from_bits, i32, normal_bits, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[300, 1, 2000, 33], [40, 20000, 7, 3000]])
def test_the_next_token_goes_on_from_what_was_kept(cuda, lens):
    B, hq, hkv = len(lens), 8, 2
    c = decode_case(cuda, lens, hq, hkv, "joint", max(lens))
    q, kp, vp, slot, off, longest = c["args"]
    _, LSE = esp.esp_partial_attn_decode_q4(*c["args"])
    sums = esp.esp_accumulate_attn_weights(q, LSE, kp, slot, off, longest, torch.zeros(kp.shape[0], device=cuda))
    kept_offsets, kept, _, freed_offsets, freed = esp.esp_evict_slots(sums, slot, off, longest, 128, keep_first=4, keep_last=16)
    stay = np.minimum(lens, 128)
    assert np.array_equal(kept_offsets.cpu().numpy(), offsets(stay))
    # the table, by the program's own indexing; then the next step's slots and lists
    table = torch.full((B, 256), -1, dtype=torch.int32, device=cuda)
    row = torch.arange(B, device=cuda).repeat_interleave(kept_offsets.diff().long())
    n = int(stay.sum())
    table[row, torch.arange(n, device=cuda) - kept_offsets[:-1].long()[row]] = kept[:n]
    taken = esp.esp_extend_block_table(table, freed[:int(freed_offsets[-1])].contiguous(), i32(stay, cuda), i32(stay + 1, cuda), 1)
    assert taken.tolist() == list(range(B + 1))
    seq_offsets, slots = esp.esp_build_slots(table, i32(stay + 1, cuda), 1, capacity=n + B)[:2]
    want = np.concatenate([np.append(kept[int(a):int(b)].cpu().numpy(), int(freed[i])) for i, (a, b) in enumerate(zip(kept_offsets[:-1], kept_offsets[1:]))])
    assert np.array_equal(seq_offsets.cpu().numpy(), offsets(stay + 1)) and np.array_equal(slots.cpu().numpy(), want)
    # its rows and its attention
    rng = np.random.default_rng(1)
    nk, nv = normal_bits(rng, B, hkv, 128), normal_bits(rng, B, hkv, 128)
    last = slots[seq_offsets[1:].long() - 1].contiguous()
    esp.esp_kv_append_q4(from_bits(nk, cuda), from_bits(nv, cuda), last, kp, vp)
    for pool, rows in (("k", nk), ("v", nv)):
        c[pool][last.cpu().numpy()] = q4.bf16_bits(q4.values(q4.quantised(rows)))
    O, LSE = esp.esp_partial_attn_decode_q4(q, kp, vp, slots, seq_offsets, 129)
    Or, Lr = oracle.partial_attn_decode_all(c["q"], c["k"], c["v"], want.astype(np.int32), offsets(stay + 1).astype(np.int32), 128 ** -0.5)
    check_o_lse(O.double().cpu().numpy().reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "the next step")
