"""The native argument checks in front of a serving step's calls: the same results, bit for bit, and the same refusals as the Python beside them."""
import pytest
import torch

from test_gpu_step import Step
from test_marshal import Plainless

pytestmark = pytest.mark.gpu


def calls(esp, cuda):
    """name -> (function, keyword arguments with everything given, the tensors that it writes)"""
    st = Step(cuda, 5)
    o, qkv = st.out, st.qkv
    return {
        "extend": (esp.esp_extend_block_table, dict(block_table=st.table, free_pages=st.free, old_lens=st.old, new_lens=st.new, page=16,
                                                    req_row=torch.arange(12, -1, -1, dtype=torch.int32, device=cuda), pages_taken=o["taken"]), ["pages_taken"]),
        "slots": (esp.esp_build_slots, dict(block_table=st.table, lens=st.old, page=16, first_token=torch.ones_like(st.old), req_row=torch.arange(13, dtype=torch.int32, device=cuda),
                                            keep_first=2, keep_last=9, pos_first=3, pos_stride=2, capacity=100, seq_offsets=o["off"], slot_idx=o["slots"],
                                            token_pos=torch.zeros(120, dtype=torch.int32, device=cuda)), ["seq_offsets", "slot_idx", "token_pos"]),
        "rotate": (esp.esp_qk_norm_rope_append, dict(q=qkv[:, :8], k=qkv[:, 8:10], v=qkv[:, 10:], q_pos=st.pos, inv_freq=st.freq, q_weight=st.w[0], k_weight=st.w[1], eps=1e-5,
                                                     interleaved=True, slot_idx=torch.arange(13, dtype=torch.int32, device=cuda), k_pool=st.pool[0], v_pool=st.pool[1],
                                                     q_out=o["q"], k_out=torch.zeros((13, 2, 128), dtype=torch.bfloat16, device=cuda),
                                                     v_out=torch.zeros((13, 2, 128), dtype=torch.bfloat16, device=cuda)), ["q_out", "k_out", "v_out"]),
        "shared": (esp.esp_partial_attn_decode_shared, dict(q=qkv[:, :8].contiguous(), k_pool=st.pool[0], v_pool=st.pool[1], prefix_slots=st.prefix_slots, prefix_offsets=st.prefix_offsets,
                                                            group_offsets=st.group_offsets, max_prefix=70, max_group=9, slot_idx=torch.arange(26, dtype=torch.int32, device=cuda),
                                                            seq_offsets=torch.arange(0, 28, 2, dtype=torch.int32, device=cuda), max_len=2, softmax_scale=None, O=o["O"], LSE=o["LSE"],
                                                            workspace=st.ws), ["O", "LSE"]),
    }


NAMES = ["extend", "slots", "rotate", "shared"]


@pytest.mark.parametrize("name", NAMES)
def test_native_checks_make_the_same_call(cuda, monkeypatch, name):
    from paper_2404_09526_amd import binding as esp
    call, kw, outs = calls(esp, cuda)[name]
    taken, marshal = [], esp._marshal

    class Spy:
        def __getattr__(self, what):
            f = getattr(marshal, what)
            return lambda *a: (taken.append(f(*a)), taken[-1])[1]
    monkeypatch.setattr(esp, "_marshal", Spy())
    results = []
    for plain in (True, False):
        first = next(iter(kw))
        for o in outs:
            kw[o].zero_()
        call(**(kw if plain else kw | {first: kw[first].as_subclass(Plainless)}))
        torch.cuda.synchronize()
        results.append([kw[o].clone() for o in outs])
    assert taken == [0, None]
    for a, b in zip(*results):
        assert a.any() and torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_what_is_not_right_is_refused(cuda, name):
    """One tensor at a time on the host, of another type, spread out, or one entry short."""
    from paper_2404_09526_amd import binding as esp
    call, kw, _ = calls(esp, cuda)[name]
    free_length = {"block_table", "free_pages", "slot_idx" if name == "shared" else "", "prefix_slots", "inv_freq", "k_pool" if name == "" else ""}
    for key, t in kw.items():
        if not isinstance(t, torch.Tensor):
            continue
        bads = [t.cpu(), torch.stack([t, t], dim=-1)[..., 0]] + ([t.to(torch.float64)] if key != "workspace" else [])
        if key not in free_length and not (name == "slots" and key in ("slot_idx", "token_pos")):
            bads.append(t[:-1].contiguous() if key != "workspace" else t[:100])
        if name == "slots" and key in ("slot_idx", "token_pos"):
            bads.append(t[:99].contiguous())
        for bad in bads:
            with pytest.raises((ValueError, esp.EspError)):
                call(**(kw | {key: bad}))
    for key in ("page", "max_prefix", "keep_last", "capacity"):
        if key in kw:
            with pytest.raises((ValueError, esp.EspError)):
                call(**(kw | {key: 1 << 32}))
            with pytest.raises((ValueError, esp.EspError)):
                call(**(kw | {key: -1}))


@pytest.mark.parametrize("name", NAMES)
def test_a_larger_output_is_written_as_far_as_the_call_goes(cuda, name):
    from paper_2404_09526_amd import binding as esp
    call, kw, outs = calls(esp, cuda)[name]
    if name == "rotate":
        return                                                       # (its outputs are asked for in the very shape)
    for o in outs:
        kw[o].zero_()
    call(**kw)
    want = {o: kw[o].clone() for o in outs}
    room = {o: torch.full((kw[o].shape[0] + 3,) + kw[o].shape[1:], 7, dtype=kw[o].dtype, device=cuda) for o in outs}
    call(**(kw | room))
    torch.cuda.synchronize()
    for o in outs:
        n = kw[o].shape[0]
        if name == "slots" and o != "seq_offsets":
            n = int(want["seq_offsets"][-1])
        assert torch.equal(room[o][:n], want[o][:n]) and (room[o][n:] == 7).all(), o
