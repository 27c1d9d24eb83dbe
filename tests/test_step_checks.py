"""What the calls of a serving step refuse, on the host, before anything is launched."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2404_09526_amd import build
    if build.is_stale():
        build.build_lib(force=True)
    from paper_2404_09526_amd import binding
    return binding


P = ctypes.c_void_p
nul, one = P(0), P(256)                                                # never dereferenced


def test_block_tables(lib):
    L, bad = lib.lib, lib.ESP_ERR_INVALID_ARG

    def extend(free=one, n_free=4, row=nul, old=one, new=one, B=2, page=16, table=one, rows=4, width=8, taken=one):
        return L.esp_extend_block_table(free, n_free, row, old, new, B, page, table, rows, width, taken, nul)
    assert extend(page=0) == bad and "page=0" in lib.last_error()
    for kw in (dict(page=-1), dict(B=-1), dict(rows=-1), dict(width=-1), dict(n_free=-1), dict(table=nul), dict(taken=nul), dict(old=nul), dict(new=nul), dict(free=nul)):
        assert extend(**kw) == bad, kw

    def slots(table=one, rows=4, width=8, page=16, row=nul, first=nul, lens=one, B=2, kf=0, kl=0, cap=10, off=one, idx=one, pos=nul):
        return L.esp_build_slots(table, rows, width, page, row, first, lens, B, kf, kl, 0, 1, cap, off, idx, pos, nul)
    for kw in (dict(page=0), dict(B=-1), dict(rows=-1), dict(width=-1), dict(table=nul), dict(lens=nul), dict(off=nul), dict(idx=nul), dict(cap=-1), dict(kf=-1, kl=4),
               dict(kl=-1), dict(kf=3)):
        assert slots(**kw) == bad, kw
    assert "window" in lib.last_error()


def test_norm_and_rotation(lib):
    L, bad = lib.lib, lib.ESP_ERR_INVALID_ARG
    far = {n: P(1 << (24 + i)) for i, n in enumerate(("q", "k", "v", "q_out", "k_out", "v_out"))}

    def call(T=4, Hq=8, Hkv=2, D=128, rot=128, inter=0, eps=1e-6, qs=1024, ks=256, vs=256, qos=1024, pos=one, freq=one, qw=nul, kw=nul, slot=one, kp=one, vp=one, S=16, **at):
        a = dict(far, **at)
        return L.esp_qk_norm_rope_append(a["q"], a["k"], a["v"], qs, ks, vs, pos, freq, rot, inter, qw, kw, ctypes.c_float(eps), T, Hq, Hkv, D, a["q_out"], qos,
                                         a["k_out"], a["v_out"], slot, kp, vp, S, nul)
    assert call(T=0) == lib.ESP_OK
    assert call(D=64, qs=512) == lib.ESP_ERR_UNSUPPORTED
    assert call(rot=24) == lib.ESP_ERR_UNSUPPORTED and "multiple of 16" in lib.last_error()
    for kw in (dict(T=-1), dict(Hq=6, Hkv=4), dict(Hkv=0), dict(rot=-2), dict(rot=130), dict(rot=7, inter=1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(qs=1016), dict(qs=1028), dict(ks=248), dict(vs=0), dict(qos=-1024), dict(qs=1 << 61), dict(pos=nul), dict(freq=nul), dict(slot=nul), dict(kp=nul), dict(vp=nul), dict(S=0), dict(S=-1),
               dict(q=nul), dict(k=nul), dict(v=nul), dict(q_out=nul), dict(q=P((1 << 24) + 8)), dict(k_out=P((1 << 27) + 2)), dict(kp=P(8)), dict(qw=P(8))):
        assert call(**kw) == bad, kw
    assert call(q_out=P((1 << 24) + 2048)) == bad and "overlaps" in lib.last_error()      # the next token's queries
    assert call(q_out=far["q"], qos=2048) == bad                       # itself, but with other strides
    assert call(q_out=P((1 << 24) + 2032), qs=2048, qos=2048) == bad   # eight elements short of the place next to it, or past it
    assert call(q_out=P((1 << 24) - 2032), qs=2048, qos=2048) == bad and call(q_out=P((1 << 24) + 2064), qs=2048, qos=2048) == bad
    assert call(k_out=far["k"], ks=512) == bad and call(v_out=P((1 << 26) + 16)) == bad


def test_decode_behind_shared_prefixes(lib):
    L, bad = lib.lib, lib.ESP_ERR_INVALID_ARG
    need = lib.esp_decode_shared_workspace_bytes(3, 2, 100, 60, 2, 10, 5, 8, 2, 128)
    assert need > 0

    def call(B=3, n_groups=2, P_total=100, max_prefix=60, max_group=2, total=10, max_len=5, Hq=8, Hkv=2, D=128, scale=0.1, q=one, kp=one, S=128, ps=one, po=one, go=one, idx=one,
             off=one, O=one, LSE=one, ws=one, ws_bytes=None):
        return L.esp_partial_attn_decode_shared(q, kp, kp, S, ps, po, go, n_groups, P_total, max_prefix, max_group, idx, off, B, total, max_len, Hq, Hkv, D, ctypes.c_float(scale), O, LSE,
                                                ws, need if ws_bytes is None else ws_bytes, nul)
    assert call(B=0, total=0, max_len=0, max_group=0) == lib.ESP_OK
    assert call(D=64) == lib.ESP_ERR_UNSUPPORTED
    for kw in (dict(B=-1), dict(n_groups=-1), dict(P_total=-1), dict(max_prefix=-1), dict(max_group=-1), dict(max_prefix=101), dict(max_group=4), dict(n_groups=0), dict(max_len=11),
               dict(Hq=6, Hkv=4), dict(q=nul), dict(kp=nul), dict(S=0), dict(ps=nul), dict(po=nul), dict(go=nul), dict(idx=nul), dict(off=nul), dict(O=nul), dict(LSE=nul),
               dict(scale=float("nan")), dict(scale=-1.0), dict(q=P(264)), dict(kp=P(258)), dict(O=P(260))):
        assert call(**kw) == bad, kw
    for kw in (dict(ws=nul), dict(ws_bytes=need - 1), dict(ws=P(264))):
        assert call(**kw) == lib.ESP_ERR_WORKSPACE, kw
    sizes = dict(B=3, n_groups=2, prefix_total=100, max_prefix=60, max_group=2, total_tokens=10, max_len=5, Hq=8, Hkv=2, D=128)
    for kw in (dict(B=-1), dict(n_groups=0), dict(prefix_total=-1), dict(max_prefix=101), dict(max_group=4), dict(total_tokens=-1), dict(Hkv=3), dict(D=64)):
        assert lib.esp_decode_shared_workspace_bytes(**dict(sizes, **kw)) == 0, kw       # the call would be refused


def test_host_tensors_and_sizes_past_32_bits_are_refused(lib):
    x = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        lib.esp_qk_norm_rope_append(x, x, x)
    with pytest.raises(ValueError, match="device memory"):
        lib.esp_extend_block_table(torch.zeros((2, 4), dtype=torch.int32), n, n, n, 1)
    with pytest.raises(ValueError, match="device memory"):
        lib.esp_build_slots(torch.zeros((2, 4), dtype=torch.int32), n, 1, capacity=4)
    with pytest.raises(ValueError, match="device memory"):
        lib.esp_partial_attn_decode_shared(x, x, x, n, n, n, 1, 1, n, n, 1)
    with pytest.raises(ValueError, match="32 bits"):
        lib._int32(1 << 31, "page")
