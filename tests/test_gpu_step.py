"""A serving step around the token pool on the GPU: block tables and slot lists from lengths, norm and rotation of new queries and keys on their
way into the pool, decode behind shared prefixes, and all of them together, against plain implementations in 64 bits (whole numbers: equal)."""
import numpy as np
import pytest
import torch

import oracle
from esp_checks import check_o_lse
from paper_2404_09526_amd import binding as esp
from paper_2404_09526_amd import workloads as wl

pytestmark = pytest.mark.gpu


def i32(x, dev):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=dev)


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


# ----------------------------------------------------------------------------------------------------------- block tables
def tables(old, new, page, rows, width, free, req_row):
    table, taken = np.full((rows, width), -7, np.int64), [0]
    for o, n, r in zip(old, new, req_row):
        a = -(-max(int(o), 0) // page)
        z = min(-(-max(int(n), 0) // page), width)
        got = max(z - a, 0) if 0 <= r < rows else 0
        for e in range(got):
            at = taken[-1] + e
            table[r, a + e] = free[at] if at < len(free) else -1
        taken.append(taken[-1] + got)
    return table, np.array(taken)


@pytest.mark.parametrize("page", [1, 5, 16])
@pytest.mark.parametrize("B", [1, 3, 64, 1023, 1024, 1025, 3000])
def test_pages_go_to_the_requests_in_order(cuda, B, page):
    rng = np.random.default_rng(B * 31 + page)
    old = rng.integers(0, 70, B)
    new = old + rng.integers(-5, 60, B)                                # some shorter: nothing
    old[rng.random(B) < 0.1] = 0
    new[rng.random(B) < 0.1] = -3
    rows, width = B + 4, 40 if page == 1 else 9                        # some past the table's width
    req_row = rng.permutation(rows)[:B]
    free = rng.permutation(100000)[:B * 20]
    want, taken = tables(old, new, page, rows, width, free, req_row)
    table = torch.full((rows, width), -7, dtype=torch.int32, device=cuda)
    got = esp.esp_extend_block_table(table, i32(free, cuda), i32(old, cuda), i32(new, cuda), page, req_row=i32(req_row, cuda))
    assert np.array_equal(got.cpu().numpy(), taken)
    assert np.array_equal(table.cpu().numpy(), want)


def test_pages_that_the_free_list_does_not_hold(cuda):
    old, new, free = [0, 4, 0, 0], [9, 40, 0, 5], [11, 12, 13, 14, 15]
    want, taken = tables(old, new, 4, 4, 16, free, range(4))
    table = torch.full((4, 16), -7, dtype=torch.int32, device=cuda)
    got = esp.esp_extend_block_table(table, i32(free, cuda), i32(old, cuda), i32(new, cuda), 4)
    assert got.tolist() == taken.tolist() and got[-1] > len(free)
    assert np.array_equal(table.cpu().numpy(), want) and (want == -1).sum() == taken[-1] - len(free)
    none = torch.empty(0, dtype=torch.int32, device=cuda)
    table.fill_(-7)
    got = esp.esp_extend_block_table(table, none, i32([0], cuda), i32([3], cuda), 1)
    assert got.tolist() == [0, 3] and table[0, :4].tolist() == [-1, -1, -1, -7]


def test_pages_rows_outside_the_table_and_no_requests(cuda):
    table = torch.full((3, 4), -7, dtype=torch.int32, device=cuda)
    got = esp.esp_extend_block_table(table, i32([5, 6, 7, 8], cuda), i32([0, 0, 0], cuda), i32([2, 2, 2], cuda), 1, req_row=i32([3, 1, -1], cuda))
    assert got.tolist() == [0, 0, 2, 2]
    assert table.tolist() == [[-7] * 4, [5, 6, -7, -7], [-7] * 4]
    none = torch.empty(0, dtype=torch.int32, device=cuda)
    assert esp.esp_extend_block_table(table, i32([5], cuda), none, none, 1).tolist() == [0]


# ----------------------------------------------------------------------------------------------------------- slot lists
def lists(table, lens, page, first, req_row, keep_first, keep_last, pos_first, pos_stride):
    off, slots, pos = [0], [], []
    for b, n in enumerate(lens):
        for t in range(max(int(first[b]), 0) if first is not None else 0, int(n)):
            if keep_last and not (t < keep_first or t >= n - keep_last):
                continue
            r, p = req_row[b], t // page
            entry = table[r, p] if 0 <= r < table.shape[0] and p < table.shape[1] else -1
            slots.append(entry * page + t % page if entry >= 0 else -1)
            pos.append(pos_first + pos_stride * t)
        off.append(len(slots))
    return np.array(off), np.array(slots, np.int64), np.array(pos, np.int64)


@pytest.mark.parametrize("keep", [(0, 0), (0, 1), (3, 17), (40, 5)], ids=["all", "last", "window", "wide-first"])
@pytest.mark.parametrize("with_first", [False, True])
@pytest.mark.parametrize("B,page", [(1, 1), (5, 16), (64, 7), (300, 1), (1025, 4), (2049, 1)])
def test_slots_of_the_requests_tokens(cuda, B, page, with_first, keep):
    rng = np.random.default_rng(B + page)
    lens = rng.integers(-2, 60, B)
    lens[rng.random(B) < 0.2] = 0
    if B == 5:
        lens[2] = 5000                                                 # one that takes more than a workgroup
    first = rng.integers(-1, 30, B) if with_first else None
    rows = B + 2
    width = max(1, -(-int(lens.max()) // page) - (1 if B == 64 else 0))   # the longest past the table's width
    req_row = rng.integers(0, rows, B)                                 # (a row may serve two requests)
    if B > 8:
        req_row[3], req_row[4] = -1, rows
    table = rng.integers(-1, 1 << 20, (rows, width))
    off, slots, pos = lists(table, lens, page, first, req_row, *keep, 5, 3)
    cap = len(slots) + 9
    idx = torch.full((cap,), -99, dtype=torch.int32, device=cuda)
    at = torch.full((cap,), -99, dtype=torch.int32, device=cuda)
    got = esp.esp_build_slots(i32(table, cuda), i32(lens, cuda), page, first_token=None if first is None else i32(first, cuda), req_row=i32(req_row, cuda),
                              keep_first=keep[0], keep_last=keep[1], pos_first=5, pos_stride=3, slot_idx=idx, token_pos=at)
    assert np.array_equal(got[0].cpu().numpy(), off)
    assert np.array_equal(idx.cpu().numpy()[:len(slots)], slots) and np.array_equal(at.cpu().numpy()[:len(slots)], pos)
    assert (idx[len(slots):] == -99).all() and (at[len(slots):] == -99).all()      # behind the list: as it was


def test_slots_a_list_longer_than_its_room_is_cut(cuda):
    table = np.arange(40).reshape(4, 10)
    lens = [4, 7, 0, 9]
    off, slots, _ = lists(table, lens, 1, None, range(4), 0, 0, 0, 1)
    for cap in (0, 1, 4, 5, 11, 19, 20):
        idx = torch.full((24,), -99, dtype=torch.int32, device=cuda)
        got = esp.esp_build_slots(i32(table, cuda), i32(lens, cuda), 1, capacity=cap, slot_idx=idx)
        assert got[0].tolist() == np.minimum(off, cap).tolist()
        assert idx.tolist() == slots[:cap].tolist() + [-99] * (24 - cap)
    # sums past 32 bits are cut, not wrapped
    got = esp.esp_build_slots(i32(table, cuda), i32([2**31 - 1] * 4, cuda), 1, capacity=3)
    assert got[0].tolist() == [0, 3, 3, 3, 3] and got[1].tolist() == [0, 1, 2]
    none = torch.empty(0, dtype=torch.int32, device=cuda)
    assert esp.esp_build_slots(i32(table, cuda), none, 1, capacity=3)[0].tolist() == [0]


def test_slots_that_lie_off_16_bytes_and_a_table_of_over_2_31_entries_apart(cuda):
    """Outputs that start inside a 16-byte piece; a table whose last row begins past 2^31 bytes."""
    rows, width = 1 << 15, (1 << 16) + 3                               # 8.6 GB
    table = torch.empty((rows, width), dtype=torch.int32, device=cuda)
    rng = np.random.default_rng(3)
    last = rng.integers(0, 1 << 20, 700)
    table[rows - 1, :700] = i32(last, cuda)
    room = torch.full((800,), -99, dtype=torch.int32, device=cuda)
    got = esp.esp_build_slots(table, i32([3, 697], cuda), 1, req_row=i32([rows - 1, rows - 1], cuda), slot_idx=room[1:702])
    assert got[0].tolist() == [0, 3, 700]
    assert np.array_equal(room.cpu().numpy()[1:701], np.concatenate([last[:3], last[:697]]))
    assert room[0] == -99 and (room[701:] == -99).all()


# ----------------------------------------------------------------------------------------------------------- norm and rotation
def rotated(x, w, pos, freq, interleaved, eps):
    """The definition in 64 bits; beside it, per element, |a| + |b| of the pair (what the errors before the last rounding go by)."""
    y = x.astype(np.float64)
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w.astype(np.float64)
    size = np.abs(y)
    if freq is not None and len(freq):
        n = len(freq)
        t = pos.astype(np.float64)[:, None, None] * freq.astype(np.float64)
        c, s = np.cos(t), np.sin(t)
        i, j = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
        a, b = y[..., i].copy(), y[..., j].copy()
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
        size[..., i] = size[..., j] = np.abs(a) + np.abs(b)
    return y, size


# Rounding to bf16: 2^-8 of the value.  Before it, in units of 2^-24 of |a| + |b|: the sum of 128 squares at most 12 (8 terms in a chain, four
# exchanges), halved by the root, root, quotient, mean and eps 4, two products 2; the reduced angle is at most pi with 1/2 unit of half a turn, pi / 2
# absolute each for its conversion and twice that for its doubling, sine and cosine 2 each; the last sum 2: below 24, taken as 32.
def close(got, want, size, what):
    err = np.abs(got.astype(np.float64) - want)
    lim = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size + 1e-37
    assert np.isfinite(got).all(), what
    assert (err <= lim).all(), f"{what}: {np.max(err / lim):.3f} x the bound"


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


LAYOUTS = [(4, 4), (1, 1), (32, 8), (12, 12), (24, 3), (7, 7), (40, 8)]
FORMS = [dict(rot=128, interleaved=False, norm="qk"), dict(rot=128, interleaved=True, norm="qk"), dict(rot=32, interleaved=False, norm=""),
         dict(rot=96, interleaved=False, norm="q"), dict(rot=20, interleaved=True, norm="k"), dict(rot=2, interleaved=True, norm=""),
         dict(rot=0, interleaved=False, norm="qk"), dict(rot=16, interleaved=False, norm="qk")]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f"rot{f['rot']}{'i' if f['interleaved'] else ''}{f['norm']}")
@pytest.mark.parametrize("T,Hq,Hkv,packed", [(n, *LAYOUTS[i % len(LAYOUTS)], bool(i & 1)) for i, n in enumerate([1, 2, 5, 33, 64, 257, 600, 1])])
def test_new_queries_and_keys(cuda, T, Hq, Hkv, packed, form):
    gen = torch.Generator(device=cuda).manual_seed(T + Hq)
    rng = np.random.default_rng(T)
    rows = torch.randn((T, Hq + 2 * Hkv, 128), generator=gen, device=cuda).bfloat16()
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    qw, kw = (torch.randn(128, generator=gen, device=cuda).bfloat16() if n in form["norm"] else None for n in "qk")
    freq = (1e4 ** (-np.arange(form["rot"] // 2) / max(1, form["rot"] // 2))).astype(np.float32)
    pos = rng.integers(0, 1 << 20, T)
    pos[0] = 2**31 - 1
    pos[-1] = 0
    slots = rng.permutation(T + 5)[:T]
    slots[rng.random(T) < 0.3] = -1
    if T > 4:
        slots[2] = T + 5                                               # outside the pool: not kept
    pools = [torch.randn((T + 5, Hkv, 128), generator=gen, device=cuda).bfloat16() for _ in range(2)]
    was = [f64(p) for p in pools]
    k_out, v_out = torch.empty((T, Hkv, 128), dtype=torch.bfloat16, device=cuda), torch.empty((T, Hkv, 128), dtype=torch.bfloat16, device=cuda)
    wq, sq = rotated(f64(q), None if qw is None else f64(qw), pos, freq, form["interleaved"], 1e-5)
    wk, sk = rotated(f64(k), None if kw is None else f64(kw), pos, freq, form["interleaved"], 1e-5)
    wv = f64(v)
    got = esp.esp_qk_norm_rope_append(q, k, v, i32(pos, cuda), torch.tensor(freq, device=cuda) if form["rot"] else None, qw, kw, 1e-5, form["interleaved"],
                                      i32(slots, cuda), pools[0], pools[1], None, k_out, v_out)
    close(f64(got[0]), wq, sq, "q")
    close(f64(k_out), wk, sk, "k")
    assert np.array_equal(f64(v_out), wv)
    kept = [t for t in range(T) if 0 <= slots[t] < T + 5]
    rest = np.setdiff1d(np.arange(T + 5), slots[kept])
    close(f64(pools[0])[slots[kept]], wk[kept], sk[kept], "pool")
    assert np.array_equal(f64(pools[1])[slots[kept]], wv[kept])
    for p, w in zip(pools, was):
        assert np.array_equal(f64(p)[rest], w[rest])                   # other rows: as they were
    assert np.array_equal(f64(pools[0])[slots[kept]], f64(k_out)[kept])   # one rounding, the same in both places
    # without dense rows, and in place: the same bits
    again = [torch.zeros_like(p) for p in pools]
    qc = q.clone() if not packed else rows.clone()[:, :Hq]
    out = esp.esp_qk_norm_rope_append(qc, k, v, i32(pos, cuda), torch.tensor(freq, device=cuda) if form["rot"] else None, qw, kw, 1e-5, form["interleaved"],
                                      i32(slots, cuda), again[0], again[1], q_out=qc)
    assert out[0] is qc and out[1] is None and torch.equal(qc, got[0])
    assert all(torch.equal(a[slots[kept]], p[slots[kept]]) for a, p in zip(again, pools))


def test_rotation_past_the_turned_elements_takes_nothing_from_others(cuda):
    """Elements past `rot` stay what they are, also next to infinities and NaN; a head's NaN stays in its pair, or with a norm in its head."""
    x = torch.ones((1, 2, 128), dtype=torch.bfloat16, device=cuda)
    x[0, 0, 3], x[0, 0, 70], x[0, 0, 100] = float("inf"), float("nan"), float("inf")
    k = torch.ones((1, 1, 128), dtype=torch.bfloat16, device=cuda)
    freq = torch.ones(32, device=cuda)
    for inter, odd in ((False, {3, 35, 70, 100}), (True, {2, 3, 70, 100})):
        q, _, _ = esp.esp_qk_norm_rope_append(x, k, k, i32([0], cuda), freq, interleaved=inter)
        bad = set((~torch.isfinite(q[0, 0])).nonzero().flatten().tolist())
        assert bad <= odd and {70, 100} <= bad, bad
        assert q[0, 0, 100] == float("inf") and torch.equal(q[0, 1], x[0, 1])
    w = torch.ones(128, dtype=torch.bfloat16, device=cuda)
    q, _, _ = esp.esp_qk_norm_rope_append(x, k, k, q_weight=w)
    assert torch.isnan(q[0, 0, 70]) and torch.isfinite(q[0, 1]).all()


def test_norm_of_zeros_and_of_the_largest_values(cuda):
    w = torch.ones(128, dtype=torch.bfloat16, device=cuda)
    x = torch.zeros((2, 1, 128), dtype=torch.bfloat16, device=cuda)
    x[1] = 1e18                                                        # its square is 1e36: the sum of 128 is still a float
    q, _, _ = esp.esp_qk_norm_rope_append(x, x, x, q_weight=w, eps=1e-6)
    assert (q[0] == 0).all() and (q[1] == 1).all()


def test_new_queries_go_next_to_the_old_ones(cuda):
    """q_out may be other columns of the buffer that q is columns of: the rows share nothing, though the two spans do."""
    gen = torch.Generator(device=cuda).manual_seed(3)
    rows = torch.randn((37, 20, 128), generator=gen, device=cuda).bfloat16()
    k = torch.randn((37, 2, 128), generator=gen, device=cuda).bfloat16()
    pos, freq = i32(np.arange(37), cuda), torch.tensor(1e4 ** (-np.arange(64) / 64), dtype=torch.float32, device=cuda)
    want, _, _ = esp.esp_qk_norm_rope_append(rows[:, 4:12], k, k, pos, freq)
    was = rows.clone()
    esp.esp_qk_norm_rope_append(rows[:, 4:12], k, k, pos, freq, q_out=rows[:, 12:])
    assert torch.equal(rows[:, 12:], want) and torch.equal(rows[:, :12], was[:, :12])
    for at in (0, 5, 11):                                              # over some of their heads
        with pytest.raises(esp.EspError, match="overlaps"):
            esp.esp_qk_norm_rope_append(rows[:, 4:12], k, k, pos, freq, q_out=rows[:, at:at + 8])


def test_rotation_of_no_tokens(cuda):
    x, y = torch.empty((0, 8, 128), dtype=torch.bfloat16, device=cuda), torch.empty((0, 2, 128), dtype=torch.bfloat16, device=cuda)
    assert esp.esp_qk_norm_rope_append(x, y, y)[0].shape == (0, 8, 128)


# ----------------------------------------------------------------------------------------------------------- decode behind shared prefixes
def shared_inputs(cuda, groups, prefixes, lens, Hq, Hkv, seed, spare=64, num_slots=None):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=cuda).manual_seed(seed)
    B, P, N = sum(groups), sum(prefixes), sum(lens)
    S = num_slots or P + N + spare
    place = rng.permutation(S)[:P + N] if S < 1 << 22 else S - 1 - rng.permutation(P + N)
    pools = []
    for _ in range(2):
        p = torch.empty((S, Hkv, 128), dtype=torch.bfloat16, device=cuda).fill_(float("nan")) if S < 1 << 22 else torch.empty((S, Hkv, 128), dtype=torch.bfloat16, device=cuda)
        p[torch.from_numpy(place.copy()).to(cuda)] = torch.randn((P + N, Hkv, 128), generator=gen, device=cuda).bfloat16()   # what no list names: NaN
        pools.append(p)
    q = torch.randn((B, Hq, 128), generator=gen, device=cuda).bfloat16()
    po, go, so = offsets(prefixes), offsets(groups), offsets(lens)
    call = dict(q=q, k_pool=pools[0], v_pool=pools[1], prefix_slots=i32(place[:P], cuda), prefix_offsets=i32(po, cuda), group_offsets=i32(go, cuda),
                max_prefix=max(prefixes, default=0), max_group=max(groups, default=0), slot_idx=i32(place[P:], cuda), seq_offsets=i32(so, cuda),
                max_len=max(lens, default=0))
    both, b = [], 0
    for g, n in enumerate(groups):
        for _ in range(n):
            both.append(np.concatenate([place[po[g]:po[g + 1]], place[P + so[b]:P + so[b + 1]]]))
            b += 1
    return call, both


def shared_reference(call, both, cuda):
    """The oracle on each request's two lists put together (rows copied out of the pools: those may be large)."""
    slots = np.concatenate(both) if both else np.zeros(0, np.int64)
    used, at = np.unique(slots, return_inverse=True)
    idx = torch.from_numpy(used.astype(np.int64)).to(cuda)
    if not len(used):
        used, idx = np.zeros(1, np.int64), torch.zeros(1, dtype=torch.int64, device=cuda)
    return oracle.partial_attn_decode_all(wl.bits(call["q"]), wl.bits(call["k_pool"][idx]), wl.bits(call["v_pool"][idx]), at.astype(np.int32),
                                          offsets([len(x) for x in both]).astype(np.int32), 128 ** -0.5)


def poisoned(nbytes, cuda):
    return torch.full((max(int(nbytes), 256),), 0xFF, dtype=torch.uint8, device=cuda)


def shared_workspace(call, cuda):
    B, Hq, D = call["q"].shape
    return poisoned(esp.esp_decode_shared_workspace_bytes(B, call["group_offsets"].numel() - 1, call["prefix_slots"].numel(), call["max_prefix"], call["max_group"],
                                                          call["slot_idx"].numel(), call["max_len"], Hq, call["k_pool"].shape[1], D), cuda)


SHARED = [
    ("one", [1], [1], [0], 4, 4), ("one-own", [1], [0], [1], 4, 4), ("nothing", [2], [0], [0, 0], 8, 2),
    ("short", [4], [300], [40, 0, 1, 77], 4, 4), ("gqa", [5], [517], [3, 64, 31, 0, 130], 32, 8), ("mqa", [3], [97], [5, 6, 7], 32, 1),
    ("mqa-wide", [9], [640], [5, 6, 7, 8, 9, 10, 11, 12, 0], 64, 1), ("odd", [7], [1000], [1] * 7, 12, 12), ("groups", [2, 1, 5], [65, 0, 400], [9, 9, 33, 0, 1, 2, 3, 4], 16, 2),
    ("empty-group", [2, 0, 3, 0], [129, 50, 31, 10], [4, 5, 6, 7, 0], 8, 8), ("no-own", [6], [255], [0] * 6, 8, 4), ("burst-2", [3, 3], [64, 1500], [100, 0, 20, 31, 32, 33], 16, 8),
    ("columns-33", [11], [700], [3] * 11, 6, 2), ("columns-64", [16], [900], [8] * 16, 32, 8), ("columns-65", [65], [333], [2] * 65, 4, 4), ("columns-128", [32], [800], [5] * 32, 32, 8),
    ("columns-200", [50], [1031], [1] * 50, 32, 8), ("columns-256", [64], [513], [7] * 64, 32, 8), ("columns-257", [257], [290], [0] * 257, 2, 2),
    ("columns-600", [150, 4], [777, 3000], [1] * 154, 8, 2), ("ragged-groups", [1, 90, 2], [4000, 33, 2100], [17] * 93, 32, 4), ("long", [2], [20000], [500, 3], 8, 2),
    ("many-groups", [1, 0, 2] * 50, [40, 7, 65] * 50, [5, 0, 33] * 50, 4, 2), ("many-requests", [699, 1], [120, 600], [0, 3, 70, 1, 600, 9, 33] * 100, 4, 1),
    ("many-of-both", [3] * 300, [1, 200, 0] * 100, [2, 0, 35] * 300, 2, 2),
]


@pytest.fixture(params=[0, 1, 2], ids=["by-estimate", "ranges", "one-launch"])
def form(request, cuda):
    """The calls in ranges and a combination, in one launch, and as the estimates say: what the tests claim, they claim of all."""
    before = esp.esp_debug_set_decode_plan(request.param)
    yield request.param
    assert esp.esp_debug_set_decode_plan(before) == request.param


@pytest.mark.parametrize("name,groups,prefixes,lens,Hq,Hkv", SHARED, ids=[s[0] for s in SHARED])
def test_decode_behind_shared_prefixes(cuda, form, name, groups, prefixes, lens, Hq, Hkv):
    call, both = shared_inputs(cuda, groups, prefixes, lens, Hq, Hkv, 11)
    Or, Lr = shared_reference(call, both, cuda)
    O = torch.full(call["q"].shape, 7.0, dtype=torch.bfloat16, device=cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, O=O, workspace=shared_workspace(call, cuda))
    D = 128
    check_o_lse(f64(O).reshape(-1, D), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, D), Lr.reshape(-1), name)
    # the same bits again, in a workspace of its own making
    O2, L2 = esp.esp_partial_attn_decode_shared(**call)
    assert torch.equal(O, O2) and torch.equal(LSE, L2)


@pytest.mark.parametrize("groups,prefixes,lens,Hq,Hkv", [([136], [20000], [7] * 136, 16, 16), ([70, 2, 9, 15, 33, 60], [16000, 320, 1120, 1600, 800, 16000], [7, 0, 40] * 63, 8, 2),
                                                         ([64], [30000], [7] * 64, 32, 8)],
                         ids=["one", "ragged", "blocks"])
@pytest.mark.parametrize("far", [None, "prefix_slots", "slot_idx"], ids=["alike", "prefix", "own"])
def test_shared_long_prefixes_of_many_columns(cuda, groups, prefixes, lens, Hq, Hkv, far):
    """The first two by eight wavefronts that have a CU alone (groups of all numbers of columns), the third by four in blocks of columns; scores of one side far above the
    other's; a NaN that stays in its head."""
    call, both = shared_inputs(cuda, groups, prefixes, lens, Hq, Hkv, 31)
    if far:
        call["k_pool"][call[far].long()] *= 40
    Or, Lr = shared_reference(call, both, cuda)
    ws = shared_workspace(call, cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=ws)
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), str(far))
    O2, L2 = esp.esp_partial_attn_decode_shared(**call)
    assert torch.equal(O, O2) and torch.equal(LSE, L2)
    if not far:
        call["k_pool"][call["prefix_slots"][12345].long(), 1] = float("nan")
        O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=ws)
        h, n = slice(Hq // Hkv, 2 * (Hq // Hkv)), groups[0]
        assert torch.isnan(LSE[:n, h]).all() and torch.isnan(O[:n, h]).all()
        O[:n, h], LSE[:n, h] = O2[:n, h], L2[:n, h]
        assert torch.equal(O, O2) and torch.equal(LSE, L2)


def test_shared_bounds_larger_than_what_is_there(cuda, form):
    call, both = shared_inputs(cuda, [3, 2], [200, 90], [5, 0, 7, 9, 1], 8, 2, 5)
    Or, Lr = shared_reference(call, both, cuda)
    call.update(max_prefix=290, max_group=5, max_len=22)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "bounds")


def test_shared_requests_past_the_stated_group_are_left_without_the_prefix(cuda, form):
    call, both = shared_inputs(cuda, [3, 40], [200, 90], [5, 0, 7] + [3] * 40, 8, 2, 41)
    for b in [2] + list(range(5, 43)):
        both[b] = both[b][200 if b < 3 else 90:]
    call["max_group"] = 2
    Or, Lr = shared_reference(call, both, cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "bounds")


def test_shared_rows_named_twice_count_twice(cuda, form):
    """In a list, in a prefix and in a request's own list, in the prefixes of two groups."""
    call, both = shared_inputs(cuda, [3, 40], [200, 90], [5, 0, 7] + [3] * 40, 8, 2, 42)
    prefix, own = call["prefix_slots"], call["slot_idx"]
    prefix[7], prefix[60:80], prefix[200:260], own[2:5], own[6] = prefix[3], prefix[150], prefix[:60], prefix[150:153], own[5]
    p, s, po, so = prefix.cpu().numpy(), own.cpu().numpy(), offsets([200, 90]), offsets([5, 0, 7] + [3] * 40)
    both = [np.concatenate([p[po[int(b >= 3)]:po[int(b >= 3) + 1]], s[so[b]:so[b + 1]]]) for b in range(43)]
    Or, Lr = shared_reference(call, both, cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "twice")


def test_shared_without_groups_is_plain_decode(cuda, form):
    call, both = shared_inputs(cuda, [3], [0], [50, 0, 7], 8, 2, 6)
    Or, Lr = shared_reference(call, both, cuda)
    none, zero = torch.empty(0, dtype=torch.int32, device=cuda), i32([0], cuda)
    call.update(prefix_slots=none, prefix_offsets=zero, group_offsets=zero, max_prefix=0, max_group=0)
    O, LSE = esp.esp_partial_attn_decode_shared(**call)
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "no groups")


def test_shared_rows_past_4_gb_of_the_pool(cuda, form):
    call, both = shared_inputs(cuda, [40, 2], [700, 130], [9] * 42, 16, 8, 9, num_slots=(1 << 22) + 5)
    Or, Lr = shared_reference(call, both, cuda)
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "far rows")


@pytest.mark.parametrize("columns", [4, 60, 120, 250])
def test_shared_nan_and_infinite_keys_show_where_they_are_seen(cuda, form, columns):
    n = columns // 2
    call, _ = shared_inputs(cuda, [n, n], [300, 310], [3] * (2 * n), 2, 2, 13)
    where = call["prefix_slots"][310].long()                           # a key of the second group's prefix
    call["k_pool"][where, 1] = float("nan")
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    assert torch.isnan(LSE[n:, 1]).all() and torch.isnan(O[n:, 1]).all()
    assert torch.isfinite(LSE[:n]).all() and torch.isfinite(LSE[n:, 0]).all() and torch.isfinite(O[:n]).all() and torch.isfinite(O[n:, 0].float()).all()
    # scores of -inf (a key of the other sign's infinity in one element) hide their key
    call, both = shared_inputs(cuda, [n], [300], [0] * n, 2, 2, 14)
    call["q"].abs_()
    call["k_pool"][call["prefix_slots"][:299].long(), :, 0] = float("-inf")
    O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
    last = call["prefix_slots"][299].long()
    s = (call["q"].double() * call["k_pool"][last].double()).sum(-1) * 128 ** -0.5
    seen = call["q"][:, :, 0] > 0
    assert torch.isfinite(LSE[seen]).all() and (LSE.double()[seen] - s[seen]).abs().max() < 1e-4 * max(1, s.abs().max())
    assert torch.equal(O[seen], call["v_pool"][last].expand_as(O)[seen])


def test_shared_scores_far_apart(cuda, form):
    """Prefix and own tokens whose scores differ by hundreds, either way: the smaller side weighs nothing and leaves no NaN."""
    for at in ("prefix_slots", "slot_idx"):
        call, both = shared_inputs(cuda, [40], [200], [33] * 40, 4, 2, 21)
        call["k_pool"][call[at].long()] *= 40
        Or, Lr = shared_reference(call, both, cuda)
        O, LSE = esp.esp_partial_attn_decode_shared(**call, workspace=shared_workspace(call, cuda))
        check_o_lse(f64(O).reshape(-1, 128), LSE.cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), at)


@pytest.fixture
def validating(cuda):
    was = esp.esp_debug_set_validate(True)
    yield
    esp.esp_debug_set_validate(was)


def test_what_the_debugging_checks_look_at(cuda, validating):
    """Refused on the host, before anything runs: slots outside the pool, offsets that decrease or end elsewhere, pieces longer than stated, rows and slots
    named twice."""
    call, _ = shared_inputs(cuda, [3, 2], [200, 90], [5, 0, 7, 9, 1], 8, 2, 5)
    esp.esp_partial_attn_decode_shared(**call)
    for name, values in (("prefix_slots", {7: 1 << 20}), ("prefix_slots", {289: -1}), ("slot_idx", {21: 1 << 20}), ("prefix_offsets", {1: 291}), ("prefix_offsets", {1: 80}),
                         ("prefix_offsets", {2: 289}), ("group_offsets", {1: 6}), ("group_offsets", {2: 4}), ("seq_offsets", {5: 21}), ("seq_offsets", {0: 1})):
        bad = call[name].clone()
        for i, x in values.items():
            bad[i] = x
        with pytest.raises(esp.EspError):
            esp.esp_partial_attn_decode_shared(**dict(call, **{name: bad}))
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=cuda)
    pools = [torch.zeros((8, 2, 128), dtype=torch.bfloat16, device=cuda) for _ in range(2)]
    esp.esp_qk_norm_rope_append(x, x, x, slot_idx=i32([3, -1, 2], cuda), k_pool=pools[0], v_pool=pools[1])
    with pytest.raises(esp.EspError, match="twice"):
        esp.esp_qk_norm_rope_append(x, x, x, slot_idx=i32([3, 1, 3], cuda), k_pool=pools[0], v_pool=pools[1])
    table, lens = torch.full((4, 3), -1, dtype=torch.int32, device=cuda), i32([1, 2], cuda)
    esp.esp_extend_block_table(table, i32([5, 6], cuda), i32([0, 0], cuda), lens, 4, req_row=i32([3, 1], cuda))
    esp.esp_build_slots(table, lens, 4, req_row=i32([3, 3], cuda), capacity=8)
    for rows in ([3, 3], [0, 4], [-1, 0]):
        with pytest.raises(esp.EspError):
            esp.esp_extend_block_table(table, i32([5, 6], cuda), i32([0, 0], cuda), lens, 4, req_row=i32(rows, cuda))
    with pytest.raises(esp.EspError):
        esp.esp_build_slots(table, lens, 4, req_row=i32([0, 4], cuda), capacity=8)


# ----------------------------------------------------------------------------------------------------------- all of them together
class Step:
    """A decoding step of a batch in two groups over a pool of pages, in a program's order: pages, slot of the new tokens, their rows, the lists, attention."""

    def __init__(self, cuda, seed=1):
        self.Hq, self.Hkv, self.page = 8, 2, 16
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=cuda).manual_seed(seed)
        self.groups, self.prefixes = [9, 4], [70, 33]
        self.own = rng.integers(1, 50, 13)                             # tokens of its own that a request has before the step
        B = 13
        pages = 400
        self.pool = [torch.randn((pages * 16, 2, 128), generator=gen, device=cuda).bfloat16() for _ in range(2)]
        place = rng.permutation(pages)
        prefix_pages, place = place[:8], place[8:]
        self.prefix = [np.concatenate([p * 16 + np.arange(16) for p in prefix_pages[:5]])[:70], np.concatenate([p * 16 + np.arange(16) for p in prefix_pages[5:]])[:33]]
        had = -(-self.own // 16)
        table = np.full((B, 8), -1, np.int64)
        for b in range(B):
            table[b, :had[b]], place = place[:had[b]], place[had[b]:]
        self.table, self.free = i32(table, cuda), i32(place, cuda)
        self.old, self.new = i32(self.own, cuda), i32(self.own + 1, cuda)
        self.pos = i32(np.repeat(self.prefixes, self.groups) + self.own, cuda)
        self.qkv = torch.randn((B, 12, 128), generator=gen, device=cuda).bfloat16()
        self.w = [torch.randn(128, generator=gen, device=cuda).bfloat16() for _ in range(2)]
        self.freq = torch.tensor(1e4 ** (-np.arange(64) / 64), dtype=torch.float32, device=cuda)
        self.prefix_slots = i32(np.concatenate(self.prefix), cuda)
        self.prefix_offsets, self.group_offsets = i32(offsets(self.prefixes), cuda), i32(offsets(self.groups), cuda)
        e = lambda *s, dt=torch.int32: torch.empty(s, dtype=dt, device=cuda)  # noqa: E731
        total = int(self.own.sum()) + B
        self.out = dict(taken=e(B + 1), new_off=e(B + 1), new_slot=e(B), off=e(B + 1), slots=e(total), q=e(B, 8, 128, dt=torch.bfloat16),
                        O=e(B, 8, 128, dt=torch.bfloat16), LSE=e(B, 8, dt=torch.float32))
        self.ws = poisoned(esp.esp_decode_shared_workspace_bytes(B, 2, 103, 70, 9, total, 51, 8, 2, 128), cuda)

    def run(self):
        o, q, k, v = self.out, self.qkv[:, :8], self.qkv[:, 8:10], self.qkv[:, 10:]
        esp.esp_extend_block_table(self.table, self.free, self.old, self.new, 16, pages_taken=o["taken"])
        esp.esp_build_slots(self.table, self.new, 16, keep_last=1, seq_offsets=o["new_off"], slot_idx=o["new_slot"])
        esp.esp_qk_norm_rope_append(q, k, v, self.pos, self.freq, *self.w, slot_idx=o["new_slot"], k_pool=self.pool[0], v_pool=self.pool[1], q_out=o["q"])
        esp.esp_build_slots(self.table, self.new, 16, seq_offsets=o["off"], slot_idx=o["slots"])
        esp.esp_partial_attn_decode_shared(o["q"], *self.pool, self.prefix_slots, self.prefix_offsets, self.group_offsets, 70, 9, o["slots"], o["off"], 51,
                                           O=o["O"], LSE=o["LSE"], workspace=self.ws)

    def check(self):
        """Against the same step in 64 bits, from the state that the run left (its new rows checked apart)."""
        table, B = self.table.cpu().numpy(), 13
        q, k, v = f64(self.qkv[:, :8]), f64(self.qkv[:, 8:10]), f64(self.qkv[:, 10:])
        pos, freq = self.pos.cpu().numpy(), self.freq.cpu().numpy()
        wq, sq = rotated(q, f64(self.w[0]), pos, freq, False, 1e-6)
        wk, sk = rotated(k, f64(self.w[1]), pos, freq, False, 1e-6)
        close(f64(self.out["q"]), wq, sq, "q")
        both = []
        for b in range(B):
            t = np.arange(self.own[b] + 1)
            own = table[b][t // 16] * 16 + t % 16
            assert (own >= 0).all()
            close(f64(self.pool[0][int(own[-1])]), wk[b], sk[b], f"key {b}")
            assert np.array_equal(f64(self.pool[1][int(own[-1])]), v[b])
            both.append(np.concatenate([self.prefix[0 if b < 9 else 1], own]))
        assert len(np.unique(np.concatenate([x[70 if b < 9 else 33:] for b, x in enumerate(both)]))) == sum(self.own) + B
        Or, Lr = shared_reference(dict(q=self.out["q"], k_pool=self.pool[0], v_pool=self.pool[1]), both, self.pool[0].device)
        check_o_lse(f64(self.out["O"]).reshape(-1, 128), self.out["LSE"].cpu().numpy().reshape(-1), Or.reshape(-1, 128), Lr.reshape(-1), "step")


def test_a_step_of_them_together(cuda):
    st = Step(cuda)
    st.run()
    st.check()


def test_a_step_captured_and_replayed(cuda):
    """Two graphs of steps with workspaces of their own, replayed in turn with new inputs and eager work between."""
    steps = [Step(cuda, 1), Step(cuda, 2)]
    graphs = []
    side = torch.cuda.Stream()
    for st in steps:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            st.run()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    for i in range(4):
        for st, g in zip(steps, graphs):
            st.qkv.copy_(torch.randn_like(st.qkv, dtype=torch.float32))
            st.out["O"].fill_(3.0)
            g.replay()
        for st in steps:
            st.check()
            kept = {k: t.clone() for k, t in st.out.items()}
            st.run()
            assert all(torch.equal(t, kept[k]) for k, t in st.out.items()), i


def test_steps_on_two_streams(cuda):
    steps = [Step(cuda, 3), Step(cuda, 4)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, s in zip(steps, streams):
            with torch.cuda.stream(s):
                st.run()
    torch.cuda.synchronize()
    for st in steps:
        st.check()
