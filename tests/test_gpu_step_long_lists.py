"""Block tables and slot lists of more elements than the launch has threads, of which a thread takes four next to each other: whole pieces of 16 bytes where they are one
request's, single ones elsewhere.  Whole numbers: equal."""
import numpy as np
import pytest
import torch

from paper_2404_09526_amd import binding as esp
from test_gpu_step import i32, offsets

pytestmark = pytest.mark.gpu

THREADS = 256 * 1536                                                   # of the largest launch for slot lists
PAGE_THREADS = 256 * 512                                               # and for block tables


def slot_lists(table, lens, page, first, req_row, keep_first, keep_last, pos_first, pos_stride):
    rows, width = table.shape
    slots, pos, counts = [], [], []
    for b, n in enumerate(lens):
        t = np.arange(max(int(first[b]), 0) if first is not None else 0, max(int(n), 0), dtype=np.int64)
        if keep_last:
            t = t[(t < keep_first) | (t >= n - keep_last)]
        entry = np.full(len(t), -1, np.int64)
        if 0 <= req_row[b] < rows:
            inside = t // page < width
            entry[inside] = table[req_row[b], t[inside] // page]
        slots.append(np.where(entry >= 0, entry * page + t % page, -1))
        pos.append(pos_first + pos_stride * t)
        counts.append(len(t))
    return offsets(counts), np.concatenate(slots), np.concatenate(pos)


@pytest.mark.parametrize("keep", [(0, 0), (5, 1001)], ids=["all", "window"])
@pytest.mark.parametrize("with_first", [False, True], ids=["", "from"])
@pytest.mark.parametrize("page", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("B", [700, 1300])
def test_long_slot_lists(cuda, B, page, with_first, keep):
    """One round of requests and one and a part; entries without a page, rows outside the table, the longest past the table's width; outputs one, two and three entries off 16
    bytes; a list that is cut inside a piece of four."""
    rng = np.random.default_rng(B + 10 * page + with_first)
    lens = rng.integers(600, 1400, B)
    lens[rng.random(B) < 0.1] = rng.integers(-1, 6)
    lens[7] = 30011
    first = rng.integers(-3, 12, B) if with_first else None
    rows, width = B + 3, -(-30011 // page) - 2
    req_row = rng.permutation(rows)[:B]
    req_row[[11, 12]] = -1, rows
    table = rng.integers(0, 1 << 24, (rows, width))
    table[rng.random((rows, width)) < 0.02] = -1
    off, slots, pos = slot_lists(table, lens, page, first, req_row, *keep, 5, 3)
    assert off[min(B, 1024)] > THREADS
    args = dict(first_token=None if first is None else i32(first, cuda), req_row=i32(req_row, cuda), keep_first=keep[0], keep_last=keep[1], pos_first=5, pos_stride=3)
    table, lens = i32(table, cuda), i32(lens, cuda)
    for shift, cap in ((1, len(slots) + 5), (2, len(slots)), (3, THREADS + 8001), (0, THREADS + 8003)):
        n = min(cap, len(slots))
        idx = torch.full((cap + 8,), -99, dtype=torch.int32, device=cuda)
        at = torch.full((cap + 8,), -99, dtype=torch.int32, device=cuda)
        got = esp.esp_build_slots(table, lens, page, capacity=cap, slot_idx=idx[shift:shift + cap], token_pos=at[shift:shift + cap], **args)
        assert np.array_equal(got[0].cpu().numpy(), np.minimum(off, cap))
        for have, want in ((idx, slots), (at, pos)):
            have = have.cpu().numpy()
            assert np.array_equal(have[shift:shift + n], want[:n]) and (have[:shift] == -99).all() and (have[shift + n:] == -99).all(), (shift, cap)


def block_table(old, new, page, rows, width, free, req_row):
    table, taken = np.full((rows, width), -7, np.int64), [0]
    for o, n, r in zip(old, new, req_row):
        a, z = -(-max(int(o), 0) // page), min(-(-max(int(n), 0) // page), width)
        got = max(z - a, 0) if 0 <= r < rows else 0
        if got:
            at = np.arange(taken[-1], taken[-1] + got)
            table[r, a:z] = np.append(free, -1)[np.minimum(at, len(free))]
        taken.append(taken[-1] + got)
    return table, np.array(taken)


@pytest.mark.parametrize("page", [1, 5, 16])
@pytest.mark.parametrize("B", [500, 1500])
@pytest.mark.parametrize("short", [0, 40003], ids=["", "free-list-short"])
def test_long_block_tables(cuda, B, page, short):
    """Prompts that are let in beside requests that have pages; a free list that ends inside a piece of four, off 16 bytes."""
    rng = np.random.default_rng(B + page + short)
    old = rng.integers(0, 90, B) * (rng.random(B) < 0.7)
    new = old + rng.integers(200, 500, B) * page
    new[rng.random(B) < 0.05] = -3
    rows, width = B + 4, 505
    req_row = rng.permutation(rows)[:B]
    req_row[9] = rows
    need = int(block_table(old, new, page, rows, width, np.zeros(0, np.int64), req_row)[1][-1])
    free = rng.permutation(need + 7)[:need + 7 - short]
    want, taken = block_table(old, new, page, rows, width, free, req_row)
    assert taken[min(B, 1024)] > PAGE_THREADS and (short == 0) == (taken[-1] <= len(free))
    table = torch.full((rows, width), -7, dtype=torch.int32, device=cuda)
    room = torch.cat([i32([-5], cuda), i32(free, cuda)])
    got = esp.esp_extend_block_table(table, room[1:], i32(old, cuda), i32(new, cuda), page, req_row=i32(req_row, cuda))
    assert np.array_equal(got.cpu().numpy(), taken) and np.array_equal(table.cpu().numpy(), want)


@pytest.mark.parametrize("n_free", [0, 1, 3, 4, 5, 255, 1021])
def test_block_tables_of_a_free_list_far_too_short(cuda, n_free):
    """The launch goes by the free list: of the 3200 entries that it does not hold a thread takes four, and they are -1."""
    rng = np.random.default_rng(n_free)
    old, new, rows = rng.integers(0, 20, 64), rng.integers(60, 90, 64), rng.permutation(70)[:64]
    free = rng.permutation(5000)[:n_free]
    want, taken = block_table(old, new, 1, 70, 80, free, rows)
    table = torch.full((70, 80), -7, dtype=torch.int32, device=cuda)
    got = esp.esp_extend_block_table(table, i32(free, cuda), i32(old, cuda), i32(new, cuda), 1, req_row=i32(rows, cuda))
    assert np.array_equal(got.cpu().numpy(), taken) and np.array_equal(table.cpu().numpy(), want)
