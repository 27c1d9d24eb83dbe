"""The operators of a serving step around the token pool, as measured: slot lists and block tables made on the GPU from request lengths, the
norm and rotation of new queries and keys on their way into the pool, and decode of batches that share a long prefix.

A case is a dict of plain values.  `prepare` makes what a serving program has in hand before the call (the outputs and workspaces that it
keeps from step to step among them), `run` is one pass: the library's call where `own` is set, else the same result by elementary torch
operations in 32 bits, rounded once.  `exact` is the definition in 64 bits.

Values are N(0, 1) in bf16, pool slots and pages a random permutation, request lengths lognormal with sigma 1 as in workloads.py.
"""
import math

import numpy as np
import torch

own = False

DIM = 128


# ----------------------------------------------------------------------------------------------------------- the cases
def slots_case(requests, median, lo, hi, page, keep_first, keep_last, stride, length_seed):
    return {"operator": "slots", "requests": requests, "median": median, "lo": lo, "hi": hi, "page": page, "keep_first": keep_first,
            "keep_last": keep_last, "pos_stride": stride, "length_seed": length_seed}


def pages_case(requests, median, lo, hi, page, added, length_seed):
    """added: tokens that every request gets beyond those it holds; 0: all of its tokens are new."""
    return {"operator": "pages", "requests": requests, "median": median, "lo": lo, "hi": hi, "page": page, "added": added,
            "length_seed": length_seed}


def rotate_case(tokens, q_heads, kv_heads, rot, interleaved, norm, packed, dense, kept, far):
    """packed: q, k, v are parts of one projection's rows; dense: K and V also leave as dense rows; kept: of 16 tokens, those whose
    slot is here; far: the position after the last token's."""
    return {"operator": "rotate", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "rot": rot, "interleaved": interleaved,
            "norm": norm, "packed": packed, "dense": dense, "kept": kept, "far": far}


def shared_case(groups, prefixes, median, lo, hi, q_heads, kv_heads, length_seed):
    return {"operator": "shared", "groups": ",".join(str(g) for g in groups), "prefixes": ",".join(str(p) for p in prefixes),
            "median": median, "lo": lo, "hi": hi, "q_heads": q_heads, "kv_heads": kv_heads, "length_seed": length_seed}


def listed():
    return [
        # the slot list of a chat service at low load: launch and latency
        dict(slots_case(16, 600, 32, 4096, 16, 0, 0, 1, 5), name="slots-16-chats"),
        # a window of 4096 behind four first tokens, positions striped over four instances, for a pass over pool rows
        dict(slots_case(64, 8192, 1024, 131072, 32, 4, 4096, 4, 2), name="slots-64-window"),
        # configuration 5's decode: 256 requests of 512 .. 1M tokens in a pool of single tokens
        dict(slots_case(256, 16384, 512, 1 << 20, 1, 0, 0, 1, 4), name="slots-256-long"),
        # the pages of one decoding step: a token each, one request in sixteen begins a page
        dict(pages_case(64, 8192, 1024, 131072, 16, 1, 2), name="pages-64-step"),
        # prompts that are let in: every token of theirs a place in a pool of single tokens
        dict(pages_case(48, 8192, 512, 65536, 1, 0, 7), name="pages-48-prompts"),
        # the smallest step there is: four tokens on four heads, rotation alone
        dict(rotate_case(4, 4, 4, 128, False, False, False, False, 16, 1024), name="rotate-4-step"),
        # a decoding step of 64 requests, grouped queries with norms, out of one projection
        dict(rotate_case(64, 32, 8, 128, False, True, True, False, 16, 131072), name="rotate-64-step"),
        # a chunk of a long prompt, its rows rotated for prefill, a quarter of them kept on this instance
        dict(rotate_case(32768, 32, 8, 128, False, True, True, True, 4, 1 << 19), name="rotate-32768-chunk"),
        # four short requests behind a short system prompt: launch and latency
        dict(shared_case([4], [300], 40, 8, 128, 4, 4, 0), name="shared-4-short"),
        # a chat service: 64 conversations behind one system prompt
        dict(shared_case([64], [2051], 600, 32, 4096, 32, 8, 5), name="shared-64-chats"),
        # sixteen questions about one long document, multi-head
        dict(shared_case([16], [65536], 300, 16, 2048, 32, 32, 6), name="shared-16-document"),
        # a batch over three documents, grouped queries
        dict(shared_case([96, 100, 60], [65549, 40000, 20011], 600, 32, 8192, 32, 8, 8), name="shared-256-documents"),
    ]


HEADS = [(4, 4), (8, 8), (8, 2), (12, 12), (16, 16), (16, 2), (24, 3), (32, 1), (32, 4), (32, 8), (32, 32), (40, 8), (64, 8)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["slots", "pages", "rotate", "shared", "shared", "shared"])
    seed = rng.randrange(1 << 20)
    if kind == "slots":
        n, median = _log(rng, 1, 512), _log(rng, 16, 16384)
        window = rng.random() < 0.4
        return slots_case(n, median, max(1, median // 16), median * 8, rng.choice([1, 1, 7, 16, 32, 64, 256]), rng.randrange(0, 9) if window else 0,
                          _log(rng, 16, 8192) if window else 0, rng.choice([1, 2, 4, 8]), seed)
    if kind == "pages":
        n, median = _log(rng, 1, 512), _log(rng, 16, 8192)
        return pages_case(n, median, max(1, median // 16), median * 4, rng.choice([1, 1, 7, 16, 64]), rng.choice([0, 1, 5, 300]), seed)
    hq, hkv = rng.choice(HEADS)
    if kind == "rotate":
        interleaved = rng.random() < 0.3
        rot = rng.choice([32, 64, 96, 128, 128]) if not interleaved else rng.choice([20, 64, 128])
        tokens = _log(rng, 1, 32768 * 48 // (hq + 2 * hkv))
        return rotate_case(tokens, hq, hkv, rot, interleaved, rng.random() < 0.6, rng.random() < 0.5, rng.random() < 0.5,
                           rng.randrange(1, 17), max(tokens, _log(rng, 1024, 1 << 20)))
    n_groups = rng.choice([1, 1, 2, 3, 5])
    groups = [_log(rng, 1, 128) for _ in range(n_groups)]
    pairs = 8e6 * 32 / hq / sum(groups)                              # query tokens x keys x heads that the largest case is not below
    longest = int(min(pairs, 131072, 2e6 / hkv / n_groups))
    prefixes = [_log(rng, 16, max(17, longest)) if rng.random() < 0.9 else 0 for _ in range(n_groups)]
    median = _log(rng, 8, max(9, min(2048, 200000 // sum(groups) * 8 // max(hkv, 8))))
    return shared_case(groups, prefixes, median, max(1, median // 8), median * 8, hq, hkv, seed)


# ----------------------------------------------------------------------------------------------------------- inputs
def _lengths(case, n):
    z = np.random.default_rng(case["length_seed"]).standard_normal(n)
    return np.clip(np.floor(np.exp(math.log(case["median"]) + z)), case["lo"], case["hi"]).astype(np.int64)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _i32(x, device="cuda"):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).to(device)


def _offsets(n):
    return np.concatenate([[0], np.cumsum(n)])


def _bf16(shape, gen):
    """N(0, 1) in bf16, drawn in pieces."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 28):
        part = flat[lo:lo + (1 << 28)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    return out


def _listed_tokens(case, lens):
    """How many tokens of each request a slot list holds."""
    if case["keep_last"] == 0:
        return lens
    return np.minimum(lens, case["keep_first"] + case["keep_last"])


def _page_lengths(case):
    old = _lengths(case, case["requests"])
    return (np.zeros_like(old), old) if case["added"] == 0 else (old, old + case["added"])


def _pages(x, page):
    return (x + page - 1) // page


def _prepare_slots(case, seed):
    lens, page = _lengths(case, case["requests"]), case["page"]
    pages = _pages(lens, page)
    n, width = len(lens), int(pages.max())
    rng = np.random.default_rng(seed)
    rows = n + 3                                                     # rows of requests that are not in this step among them
    table = np.full((rows, width), -1, np.int64)
    req_row = rng.permutation(rows)[:n]
    place = rng.permutation(int(pages.sum()) + 64)
    at = _offsets(pages)
    for b in range(n):
        table[req_row[b], :pages[b]] = place[at[b]:at[b + 1]]
    total = int(_listed_tokens(case, lens).sum())
    window = case["keep_last"] > 0
    return {"case": case, "table": _i32(table), "req_row": _i32(req_row), "lens": _i32(lens), "total": total,
            "offsets": torch.empty(n + 1, dtype=torch.int32, device="cuda"), "slots": torch.empty(total, dtype=torch.int32, device="cuda"),
            "pos": torch.empty(total, dtype=torch.int32, device="cuda") if window else None}


def _prepare_pages(case, seed):
    old, new = _page_lengths(case)
    page, n = case["page"], len(old)
    rng = np.random.default_rng(seed)
    had, will = _pages(old, page), _pages(new, page)
    taken = int((will - had).sum())
    place = rng.permutation(int(will.sum()) + 256)
    table = np.full((n + 2, int(will.max()) + 4), -1, np.int64)
    req_row = rng.permutation(n + 2)[:n]
    at = _offsets(had)
    for b in range(n):
        table[req_row[b], :had[b]] = place[at[b]:at[b + 1]]
    return {"case": case, "table": _i32(table), "req_row": _i32(req_row), "old": _i32(old), "new": _i32(new), "free": _i32(place[int(had.sum()):]),
            "total": taken, "taken": torch.empty(n + 1, dtype=torch.int32, device="cuda")}


def _prepare_rotate(case, seed):
    T, hq, hkv = case["tokens"], case["q_heads"], case["kv_heads"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    if case["packed"]:
        rows = _bf16((T, hq + 2 * hkv, DIM), gen)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    else:
        q, k, v = _bf16((T, hq, DIM), gen), _bf16((T, hkv, DIM), gen), _bf16((T, hkv, DIM), gen)
    weights = [1 + 0.1 * torch.randn(DIM, generator=gen, device="cuda") for _ in range(2)]
    q_weight, k_weight = (w.to(torch.bfloat16) for w in weights) if case["norm"] else (None, None)
    half = case["rot"] // 2
    inv_freq = torch.tensor(1e6 ** (-np.arange(half) / half), dtype=torch.float32, device="cuda")
    if T <= 512:                                                     # a token of each request
        pos = rng.integers(0, case["far"], T)
    else:
        pos = np.arange(case["far"] - T, case["far"])
    kept = rng.permutation(T)[:max(1, T * case["kept"] // 16)]
    pool = len(kept) + len(kept) // 4 + 8
    slot = np.full(T, -1, np.int64)
    slot[kept] = rng.permutation(pool)[:len(kept)]
    kept = np.sort(kept)
    new = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    return {"case": case, "q": q, "k": k, "v": v, "q_weight": q_weight, "k_weight": k_weight, "inv_freq": inv_freq, "pos": _i32(pos),
            "slot": _i32(slot), "kept": torch.from_numpy(kept).cuda(), "kept_slot": torch.from_numpy(slot[kept]).cuda(),
            "k_pool": _bf16((pool, hkv, DIM), gen), "v_pool": _bf16((pool, hkv, DIM), gen), "q_out": new(T, hq, DIM),
            "k_out": new(T, hkv, DIM) if case["dense"] else None, "v_out": new(T, hkv, DIM) if case["dense"] else None}


def _shared_sizes(case):
    groups, prefixes = np.array(_ints(case["groups"])), np.array(_ints(case["prefixes"]))
    return groups, prefixes, _lengths(case, int(groups.sum()))


def _prepare_shared(case, seed):
    hq, hkv = case["q_heads"], case["kv_heads"]
    groups, prefixes, lens = _shared_sizes(case)
    B, P, N = int(groups.sum()), int(prefixes.sum()), int(lens.sum())
    gen = torch.Generator(device="cuda").manual_seed(seed)
    place = np.random.default_rng(seed).permutation(P + N + (P + N) // 8 + 16)
    st = {"case": case, "q": _bf16((B, hq, DIM), gen), "k_pool": _bf16((len(place), hkv, DIM), gen), "v_pool": _bf16((len(place), hkv, DIM), gen),
          "prefix_slots": _i32(place[:P]), "prefix_offsets": _i32(_offsets(prefixes)), "group_offsets": _i32(_offsets(groups)),
          "slot_idx": _i32(place[P:P + N]), "seq_offsets": _i32(_offsets(lens)), "max_prefix": int(prefixes.max()), "max_group": int(groups.max()),
          "max_len": int(lens.max()), "scale": DIM ** -0.5, "O": torch.empty((B, hq, DIM), dtype=torch.bfloat16, device="cuda"),
          "LSE": torch.empty((B, hq), dtype=torch.float32, device="cuda"), "groups": [int(x) for x in groups],
          "prefixes": [int(x) for x in prefixes], "lens": [int(x) for x in lens]}
    if own:
        from paper_2404_09526_amd import binding as esp
        st["workspace"] = torch.empty(max(256, esp.esp_decode_shared_workspace_bytes(B, len(groups), P, st["max_prefix"], st["max_group"], N,
                                                                                     st["max_len"], hq, hkv, DIM)), dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    return {"slots": _prepare_slots, "pages": _prepare_pages, "rotate": _prepare_rotate, "shared": _prepare_shared}[case["operator"]](case, seed)


# ----------------------------------------------------------------------------------------------------------- the plain forms
def _plain_slots(st):
    c = st["case"]
    lens = st["lens"].long()
    head, tail = c["keep_first"], c["keep_last"]
    n = lens if tail == 0 else lens.clamp(max=head + tail)
    offsets = torch.zeros(len(lens) + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = n.cumsum(0)
    b = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n, output_size=st["total"])
    i = torch.arange(st["total"], device="cuda") - offsets[b]
    if tail:
        i = torch.where(i < head, i, i + (lens - n)[b])
    page = c["page"]
    slots = st["table"][st["req_row"].long()[b], i // page].long() * page + i % page
    pos = 1 + i * c["pos_stride"]
    return offsets.int(), slots.int(), pos.int() if tail else None


def _plain_pages(st):
    page = st["case"]["page"]
    had, will = _pages(st["old"].long(), page), _pages(st["new"].long(), page)
    n = will - had
    taken = torch.zeros(len(n) + 1, dtype=torch.int64, device="cuda")
    taken[1:] = n.cumsum(0)
    b = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=st["total"])
    j = torch.arange(st["total"], device="cuda")
    st["table"][st["req_row"].long()[b], had[b] + j - taken[b]] = st["free"][j]
    return st["table"], taken.int()


def _plain_rotate(st):
    c = st["case"]
    half = c["rot"] // 2
    turn = st["pos"].double()[:, None] * st["inv_freq"].double()     # far positions: in 32 bits an angle would be off by a tenth
    cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]

    def rotated(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        out = x.clone()
        if c["interleaved"]:
            a, b = x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]
            out[..., 0:c["rot"]:2], out[..., 1:c["rot"]:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            out[..., :half], out[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
        return out.bfloat16()

    q, k = rotated(st["q"], st["q_weight"]), rotated(st["k"], st["k_weight"])
    st["k_pool"][st["kept_slot"]] = k[st["kept"]]
    st["v_pool"][st["kept_slot"]] = st["v"][st["kept"]]
    return q, st["k_pool"], st["v_pool"], k if c["dense"] else None, st["v"].contiguous() if c["dense"] else None


def _plain_shared(st):
    c = st["case"]
    hq, hkv = c["q_heads"], c["kv_heads"]
    G = hq // hkv
    q = st["q"].float() * st["scale"]
    O, LSE = torch.empty_like(st["O"]), torch.empty_like(st["LSE"])

    def part(rows, k, v):
        """rows [n, 128] against k, v [m, 128]: sums against the maximum."""
        s = rows @ k.t()
        m = s.max(1, keepdim=True).values
        p = torch.exp(s - m)
        return m, p.sum(1, keepdim=True), p @ v

    b0 = p0 = t0 = 0
    for n, P in zip(st["groups"], st["prefixes"]):
        shared = []
        if P:
            slots = st["prefix_slots"][p0:p0 + P].long()
            k, v = st["k_pool"][slots].float(), st["v_pool"][slots].float()
            for h in range(hkv):
                rows = q[b0:b0 + n, h * G:(h + 1) * G].reshape(n * G, DIM)
                shared.append([x.view(n, G, -1) for x in part(rows, k[:, h], v[:, h])])
            m, l, o = (torch.stack(x, 1) for x in zip(*shared))      # [n, Hkv, G, .]
        for j in range(n):
            L, b = st["lens"][b0 + j], b0 + j
            slots = st["slot_idx"][t0:t0 + L].long()
            k, v = st["k_pool"][slots].float().permute(1, 0, 2), st["v_pool"][slots].float().permute(1, 0, 2)
            s = torch.matmul(q[b].view(hkv, G, DIM), k.transpose(1, 2).contiguous())
            top = s.max(-1, keepdim=True).values
            if P:
                top = torch.maximum(top, m[j])
            p = torch.exp(s - top)
            total, out = p.sum(-1, keepdim=True), torch.matmul(p, v.contiguous())
            if P:
                w = torch.exp(m[j] - top)
                total, out = total + w * l[j], out + w * o[j]
            O[b] = (out / total).reshape(hq, DIM)
            LSE[b] = (top + total.log()).view(hq)
            t0 += L
        b0, p0 = b0 + n, p0 + P
    return O, LSE


# ----------------------------------------------------------------------------------------------------------- one pass
def run(state):
    c, st = state["case"], state
    if not own:
        return {"slots": _plain_slots, "pages": _plain_pages, "rotate": _plain_rotate, "shared": _plain_shared}[c["operator"]](st)
    from paper_2404_09526_amd import binding as esp
    if c["operator"] == "slots":
        return esp.esp_build_slots(st["table"], st["lens"], c["page"], req_row=st["req_row"], keep_first=c["keep_first"], keep_last=c["keep_last"],
                                   pos_first=1, pos_stride=c["pos_stride"], seq_offsets=st["offsets"], slot_idx=st["slots"], token_pos=st["pos"])
    if c["operator"] == "pages":
        taken = esp.esp_extend_block_table(st["table"], st["free"], st["old"], st["new"], c["page"], req_row=st["req_row"], pages_taken=st["taken"])
        return st["table"], taken
    if c["operator"] == "rotate":
        q, k, v = esp.esp_qk_norm_rope_append(st["q"], st["k"], st["v"], st["pos"], inv_freq=st["inv_freq"], q_weight=st["q_weight"],
                                              k_weight=st["k_weight"], eps=1e-6, interleaved=c["interleaved"], slot_idx=st["slot"],
                                              k_pool=st["k_pool"], v_pool=st["v_pool"], q_out=st["q_out"], k_out=st["k_out"], v_out=st["v_out"])
        return q, st["k_pool"], st["v_pool"], k, v
    return esp.esp_partial_attn_decode_shared(st["q"], st["k_pool"], st["v_pool"], st["prefix_slots"], st["prefix_offsets"], st["group_offsets"],
                                              st["max_prefix"], st["max_group"], st["slot_idx"], st["seq_offsets"], st["max_len"],
                                              softmax_scale=st["scale"], O=st["O"], LSE=st["LSE"], workspace=st["workspace"])


# ----------------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["operator"] == "slots":
        lens = _lengths(case, case["requests"])
        n = _listed_tokens(case, lens)
        total, pages = int(n.sum()), int(_pages(n, case["page"]).sum())
        return {"bytes": 4 * (total * (2 if case["keep_last"] else 1) + pages + 3 * len(lens)), "flops": 0}
    if case["operator"] == "pages":
        old, new = _page_lengths(case)
        return {"bytes": 4 * (2 * int((_pages(new, case["page"]) - _pages(old, case["page"])).sum()) + 4 * len(old)), "flops": 0}
    hq, hkv = case["q_heads"], case["kv_heads"]
    if case["operator"] == "rotate":
        T, row = case["tokens"], 2 * DIM
        kept = max(1, T * case["kept"] // 16)
        written = T * hq + 2 * hkv * (kept + (T if case["dense"] else 0))
        read = T * hq + 2 * hkv * (T if case["dense"] else kept)
        norm = 4 if case["norm"] else 0
        return {"bytes": row * (read + written) + 8 * T, "flops": T * (hq + hkv) * (3 * case["rot"] + norm * DIM)}
    groups, prefixes, lens = _shared_sizes(case)
    rows = int(prefixes.sum() + lens.sum())
    return {"bytes": rows * (hkv * 4 * DIM + 4) + int(groups.sum()) * hq * (4 * DIM + 4),
            "flops": 4 * DIM * hq * int((groups * prefixes).sum() + lens.sum())}


# ----------------------------------------------------------------------------------------------------------- the definitions
def _exact_slots(case, st):
    lens, rows, table = st["lens"].cpu().numpy(), st["req_row"].cpu().numpy(), st["table"].cpu().numpy().astype(np.int64)
    slots, pos, counts = [], [], []
    for L, r in zip(lens, rows):
        i = np.arange(L, dtype=np.int64)
        if case["keep_last"]:
            i = i[(i < case["keep_first"]) | (i >= L - case["keep_last"])]
        slots.append(table[r][i // case["page"]] * case["page"] + i % case["page"])
        pos.append(1 + i * case["pos_stride"])
        counts.append(len(i))
    return _i32(_offsets(counts)), _i32(np.concatenate(slots)), _i32(np.concatenate(pos)) if case["keep_last"] else None


def _exact_pages(case, st):
    old, new, rows = (st[x].cpu().numpy() for x in ("old", "new", "req_row"))
    table, free, taken = st["table"].cpu().numpy(), st["free"].cpu().numpy(), [0]
    for o, n, r in zip(old, new, rows):
        a, z = -(-int(o) // case["page"]), -(-int(n) // case["page"])
        table[r, a:z] = free[taken[-1]:taken[-1] + z - a]
        taken.append(taken[-1] + max(z - a, 0))
    return _i32(table), _i32(np.array(taken))


def _exact_rotate(case, st):
    half = case["rot"] // 2
    angle = st["pos"].double().view(-1, 1, 1) * st["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)                # unit complex numbers: a pair of elements is turned by a product

    def turned(x, w):
        y = x.double()
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / DIM + 1e-6).sqrt() * w.double()
        r = y[..., :case["rot"]]
        z = torch.complex(r[..., 0::2].contiguous(), r[..., 1::2].contiguous()) if case["interleaved"] else torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous())
        z = z * turn
        r = torch.stack([z.real, z.imag], -1).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([r, y[..., case["rot"]:]], -1)

    k_pool, v_pool = st["k_pool"].double(), st["v_pool"].double()
    k = turned(st["k"], st["k_weight"])
    keep = st["slot"] >= 0
    k_pool[st["slot"][keep].long()] = k[keep]
    v_pool[st["slot"][keep].long()] = st["v"].double()[keep]
    return turned(st["q"], st["q_weight"]), k_pool, v_pool, k if case["dense"] else None, st["v"].double() if case["dense"] else None


def _exact_shared(case, st):
    hq, hkv = case["q_heads"], case["kv_heads"]
    G = hq // hkv
    O = torch.empty((len(st["lens"]), hq, DIM), dtype=torch.float64, device="cuda")
    LSE = torch.empty((len(st["lens"]), hq), dtype=torch.float64, device="cuda")
    b = p = t = 0
    for n, P in zip(st["groups"], st["prefixes"]):
        for _ in range(n):
            rows = torch.cat([st["prefix_slots"][p:p + P], st["slot_idx"][t:t + st["lens"][b]]]).long()
            for h in range(hkv):
                x = st["q"][b, h * G:(h + 1) * G].double() @ st["k_pool"][rows, h].double().t().contiguous() * st["scale"]
                LSE[b, h * G:(h + 1) * G] = torch.logsumexp(x, 1)
                O[b, h * G:(h + 1) * G] = torch.softmax(x, 1) @ st["v_pool"][rows, h].double()
            t, b = t + st["lens"][b], b + 1
        p += P
    return O, LSE


def exact(case, seed):
    st = prepare(case, seed)
    return {"slots": _exact_slots, "pages": _exact_pages, "rotate": _exact_rotate, "shared": _exact_shared}[case["operator"]](case, st)
