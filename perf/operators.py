"""The operators of serving from a cache of keys and values in 8 bits, over the range in which they are called.

A serving process keeps keys and values in pages of 64 tokens, one e4m3 code per value and one fp32 scale for each page and
head.  A step of it gives every request's new tokens their places (block tables and slot maps from the lengths, on the GPU),
writes the new keys and values there, and attends over the cache: one query row per request (decode), a few (a drafted
continuation) or a chunk of a prompt.

Cases are dicts; their lengths follow from the case alone, so the work of a case does not depend on the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
FLOOR = 2.0 ** -100                 # the smallest scale that an append writes


# ---- cases -----------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # Places for one decode step of a rank's 64 requests: a token each, every 64th on a new page.
        dict(name="slots_step", op="slots", batch=64, lens="uniform", low=1024, high=8192, new="one", new_high=1, spare=64, pad=0, short=0),
        # Places for a step that mixes 512 requests' decode tokens and prompt chunks of up to 1,024 tokens, into padded
        # buffers; the free list ends before the last requests are served.
        dict(name="slots_mixed", op="slots", batch=512, lens="log", low=16, high=32768, new="mixed", new_high=1024, spare=64, pad=1000, short=1),
        # Keys and values of that decode step: 64 rows of eight heads, most of them into a page that is partly full.
        dict(name="append_step", op="append", batch=64, lens="uniform", low=256, high=2048, new="one", new_high=1, kv_heads=8, dim=128, dtype="bf16"),
        # A rank's shard of a rollout step, one head of 64, fp16, ragged chunks that begin anywhere in a page.
        dict(name="append_ragged", op="append", batch=37, lens="log", low=1, high=4096, new="mixed", new_high=500, kv_heads=3, dim=64, dtype="fp16"),
        # Four prompts of 8,192 tokens at once.
        dict(name="append_prompts", op="append", batch=4, lens="fixed", low=0, high=0, new="fixed", new_high=8192, kv_heads=8, dim=128, dtype="bf16"),
        # The smallest decode batch: contexts of 1, 17, 64 and 200 tokens.  Launches and host work are all there is.
        dict(name="decode_tiny", op="attention", batch=4, lens="1,17,64,200", low=1, high=200, heads=16, kv_heads=2, dim=128, dtype="bf16", rows="one", rows_high=1),
        # One decode step of a rank's 64 requests, all heads, contexts of 1k to 8k tokens.
        dict(name="decode_batch", op="attention", batch=64, lens="uniform", low=1024, high=8192, heads=64, kv_heads=8, dim=128, dtype="bf16", rows="one", rows_high=1),
        # RL rollout on a rank that owns one key head: 512 requests, many short and a few very long.
        dict(name="decode_rollout", op="attention", batch=512, lens="rollout", low=16, high=32768, heads=8, kv_heads=1, dim=128, dtype="bf16", rows="one", rows_high=1),
        # One very long context: few rows, the work is split over the tokens.
        dict(name="decode_long", op="attention", batch=1, lens="fixed", low=262144, high=262144, heads=64, kv_heads=8, dim=128, dtype="bf16", rows="one", rows_high=1),
        # Drafted continuations: up to 8 causal rows per request, heads of 64, fp16.
        dict(name="draft_rows", op="attention", batch=29, lens="uniform", low=1000, high=8000, heads=12, kv_heads=4, dim=64, dtype="fp16", rows="ragged", rows_high=8),
        # Chunks of 2,048 prompt rows behind contexts that are in the cache already.
        dict(name="chunk_prompts", op="attention", batch=2, lens="fixed", low=8192, high=8192, heads=32, kv_heads=8, dim=128, dtype="bf16", rows="fixed", rows_high=2048),
        # A mixed step: odd chunks beside requests that decode one row.
        dict(name="chunk_mixed", op="attention", batch=13, lens="log", low=800, high=9001, heads=16, kv_heads=2, dim=128, dtype="fp16", rows="mixed", rows_high=777),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most = [work(c) for c in listed()]
    bytes_most, flops_most = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        op = rng.choice(["slots", "append", "append", "attention", "attention", "attention", "attention"])
        c = dict(op=op, batch=_log(rng, 1, 512), lens=rng.choice(["uniform", "log", "rollout"]), low=_log(rng, 1, 2000))
        c["high"] = _log(rng, c["low"], 32768)
        if op == "slots":
            c.update(new=rng.choice(["one", "mixed", "ragged"]), new_high=_log(rng, 1, 2048), spare=rng.randrange(0, 200), pad=rng.randrange(0, 2000), short=rng.randrange(2))
        else:
            c.update(kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([64, 128]), dtype=rng.choice(["bf16", "fp16"]))
        if op == "append":
            c["high"] = min(c["high"], 4096)
            c["low"] = min(c["low"], c["high"])
            c.update(new=rng.choice(["one", "mixed", "ragged"]), new_high=_log(rng, 1, 4096))
        if op == "attention":
            c["heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 16])
            kind = rng.choice(["one", "one", "few", "chunk"])
            if kind == "one":
                c.update(rows="one", rows_high=1)
            elif kind == "few":
                c.update(rows=rng.choice(["fixed", "ragged"]), rows_high=rng.randrange(2, 9))
            else:
                c["batch"] = _log(rng, 1, 16)
                c.update(rows=rng.choice(["fixed", "ragged", "mixed"]), rows_high=_log(rng, 9, 2048))
            c["low"] = max(c["low"], c["rows_high"])
            c["high"] = max(c["high"], c["low"])
        w = work(c)
        if w["bytes"] > bytes_most or w["flops"] > flops_most:
            continue
        if op == "attention":
            dense = c["batch"] * max(_lens(c))
            if dense * c["kv_heads"] * c["dim"] <= 512 * 32768 * 128 and dense * c["heads"] * c["rows_high"] <= 2 * 32 * 2048 * 8192:
                return c
        elif sum(_lens(c)) + sum(_new(c)) <= 2_000_000:
            if op == "slots" or (sum(_lens(c)) + sum(_new(c))) * c["kv_heads"] * c["dim"] <= 200_000 * 1024:
                return c


def _lens(c):
    """Tokens of each request that are in the cache (attention: with the query rows' own)."""
    if "," in c["lens"]:
        return [int(x) for x in c["lens"].split(",")]
    g = np.random.default_rng([c["batch"], c["low"], c["high"]])
    if c["lens"] == "fixed":
        x = np.full(c["batch"], c["low"])
    elif c["lens"] == "uniform":
        x = g.integers(c["low"], c["high"] + 1, c["batch"])
    elif c["lens"] == "log":
        x = np.exp(g.uniform(math.log(c["low"]), math.log(c["high"]), c["batch"])).round()
    else:                                       # rollout: lognormal around 2,048
        x = np.clip(np.exp(g.normal(math.log(2048), 1.2, c["batch"])).round(), c["low"], c["high"])
    return [int(v) for v in x]


def _counts(kind, high, batch):
    g = np.random.default_rng([batch, high, 7])
    if kind in ("one", "fixed"):
        return [1 if kind == "one" else high] * batch
    if kind == "ragged":
        return [int(v) for v in g.integers(1, high + 1, batch)]
    x = g.integers(1, high + 1, batch)          # mixed: most requests decode one token, a third bring a chunk
    return [int(v) if k % 3 == 0 else 1 for k, v in enumerate(x)]


def _new(c):
    return _counts(c["new"], c["new_high"], c["batch"])


def _rows(c):
    return _counts(c["rows"], c["rows_high"], c["batch"])


def _pages(n):
    return -(-n // PAGE)


def work(c):
    lens, B = _lens(c), c["batch"]
    if c["op"] == "slots":
        new = _new(c)
        fresh = sum(_pages(a + b) - _pages(a) for a, b in zip(lens, new))
        # lengths read, sums and new lengths written, a free page read and an entry written for each new page, a slot and a
        # position for each place
        return {"bytes": 4 * (2 * B + 2 * B + 1) + 8 * fresh + 12 * (sum(new) + c["pad"]) + 4 * B, "flops": 0}
    if c["op"] == "append":
        new = _new(c)
        row = c["kv_heads"] * c["dim"]
        pages = sum(_pages(a + b) - a // PAGE for a, b in zip(lens, new))
        return {"bytes": 2 * sum(new) * row * 3 + 8 * sum(new) + 2 * 4 * pages * c["kv_heads"], "flops": 2 * 2 * sum(new) * row}
    rows, D, heads, kv = _rows(c), c["dim"], c["heads"], c["kv_heads"]
    seen = sum(r * n - r * (r - 1) // 2 for r, n in zip(rows, lens))
    pages = sum(_pages(n) for n in lens)
    return {"bytes": 2 * sum(lens) * kv * D + pages * (8 * kv + 4) + sum(rows) * heads * (4 * D + 4) + 8 * B, "flops": 4 * D * heads * seen}


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _table(lens, g, spare_entries=0):
    """Block table [B][W] over a pool with a quarter more pages than are used, in random order; entries that name no page of a
    request hold -1.  Returns (table, pool pages, the pages not used)."""
    pages = [_pages(n) for n in lens]
    total = sum(pages)
    pool = total + total // 4 + 8
    order = g.permutation(pool).astype(np.int32)
    table = np.full((len(lens), max(max(pages), 1) + spare_entries), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    return table, pool, order[at:]


def _slots_of(table, lens, new):
    """slot = page * 64 + offset of each new token, request after request."""
    out = []
    for i, (a, b) in enumerate(zip(lens, new)):
        t = np.arange(a, a + b)
        out.append(table[i, t // PAGE].astype(np.int64) * PAGE + t % PAGE)
    return np.concatenate(out)


def _codes(shape, gen):
    """e4m3 codes of normal values whose largest use the range of the format."""
    out = torch.empty(shape, dtype=E4M3, device="cuda")
    for part in torch.split(out, max(1, 2 ** 26 // max(1, out[0].numel()))):
        part.copy_((torch.randn(part.shape, device="cuda", generator=gen) * 100).clamp_(-448, 448))
    return out


def _scales(shape, gen):
    return torch.exp2(torch.randint(-8, -5, shape, device="cuda", generator=gen).float())


def _int(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def prepare(case, seed):
    c = case
    g, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    lens = _lens(c)
    if c["op"] == "slots":
        new = _new(c)
        lens = [int(v) for v in g.permutation(lens)]        # which request is how long differs from seed to seed
        fresh = sum(_pages(a + b) - _pages(a) for a, b in zip(lens, new))
        table, pool, free = _table(lens, g, _pages(c["new_high"]) + 1)
        more = np.arange(pool, pool + fresh + c["spare"], dtype=np.int32)
        free = g.permutation(np.concatenate([free, more]))
        begin = 3
        if c["short"]:
            free = free[:begin + max(0, fresh - fresh // 8)]
        return dict(c, block_table=_int(table), seq_lens=_int(lens), new_lens=_int(new), free_pages=_int(free), free_begin=_int([begin]), num_slots=sum(new) + c["pad"])
    if c["op"] == "append":
        new = _new(c)
        table, pool, _ = _table([a + b for a, b in zip(lens, new)], g)
        shape = (sum(new), c["kv_heads"], c["dim"])
        loud = torch.exp2(torch.randint(-2, 3, (shape[0], shape[1], 1), device="cuda", generator=gen).float())
        kv = [(torch.randn(shape, device="cuda", generator=gen) * loud).to(TYPES[c["dtype"]]) for _ in range(2)]
        pools = [_codes((pool, c["kv_heads"], PAGE, c["dim"]), gen) for _ in range(2)]
        scales = [_scales((pool, c["kv_heads"]), gen) for _ in range(2)]
        first = np.concatenate([[0], np.cumsum(new)[:-1]])
        return dict(c, k=kv[0], v=kv[1], slot_map=torch.tensor(_slots_of(table, lens, new), device="cuda"), first=torch.tensor(first, device="cuda"),
                    k_pool=pools[0], v_pool=pools[1], k_scales=scales[0], v_scales=scales[1])
    rows = _rows(c)
    table, pool, free = _table(lens, g)
    pools = [_codes((pool, c["kv_heads"], PAGE, c["dim"]), gen) for _ in range(2)]
    scales = [_scales((pool, c["kv_heads"]), gen) for _ in range(2)]
    for p in pools:                            # what lies behind a request's last token, and on pages of no request, may be anything
        raw = p.view(torch.uint8)
        raw[torch.tensor(free.astype(np.int64), device="cuda")] = 0x7F
        last = torch.tensor([table[i, (n - 1) // PAGE] for i, n in enumerate(lens)], device="cuda").long()
        used = torch.tensor([(n - 1) % PAGE + 1 for n in lens], device="cuda")
        tail = raw[last]
        raw[last] = torch.where(torch.arange(PAGE, device="cuda")[None, None, :, None] >= used[:, None, None, None], torch.full_like(tail, 0x7F), tail)
    q = torch.randn((sum(rows), c["heads"], c["dim"]), device="cuda", generator=gen).to(TYPES[c["dtype"]])
    q_start = _int(np.concatenate([[0], np.cumsum(rows)])) if c["rows"] != "one" else None
    return dict(c, q=q, q_start=q_start, max_rows=max(rows), k_pool=pools[0], v_pool=pools[1], k_scales=scales[0], v_scales=scales[1],
                block_table=_int(table), seq_lens=_int(lens), scale=1.0 / math.sqrt(c["dim"]))


# ---- one pass --------------------------------------------------------------------------------------------------------------

def run(s):
    return {"slots": _run_slots, "append": _run_append, "attention": _run_attention}[s["op"]](s)


def _run_slots(s):
    if own:
        from paper_2609_37626_b200 import binding
        slot_map, positions, q_start, new_seq_lens, counts = binding.splash_kv_slots(s["block_table"], s["seq_lens"], s["new_lens"], s["free_pages"],
                                                                                     s["free_begin"], s["num_slots"])
    else:
        slot_map, positions, q_start, new_seq_lens, counts = _plain_slots(s["block_table"], s["seq_lens"], s["new_lens"], s["free_pages"], s["free_begin"],
                                                                          s["num_slots"])
    return {"block_table": s["block_table"], "slot_map": slot_map, "positions": positions, "q_start": q_start, "new_seq_lens": new_seq_lens, "counts": counts}


def _plain_slots(table, lens, new, free, begin, num_slots):
    B, W = table.shape
    dev = table.device
    start = torch.zeros(B + 1, dtype=torch.int64, device=dev)
    start[1:] = torch.cumsum(new, 0)
    have, want = (lens.long() + PAGE - 1) // PAGE, (lens.long() + new + PAGE - 1) // PAGE
    fits = (want <= W) & (start[1:] <= num_slots)
    need = torch.where(fits, want - have, 0)
    upto = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (upto <= free.numel() - begin.long()))
    j = torch.arange(W, device=dev)[None]
    fresh = served[:, None] & (j >= have[:, None]) & (j < want[:, None])
    at = begin.long() + (upto - need)[:, None] + j - have[:, None]
    table.copy_(torch.where(fresh, free[at.clamp(0, max(free.numel() - 1, 0))], table))
    t = torch.arange(num_slots, device=dev)
    i = torch.searchsorted(start, t, right=True) - 1
    i_ = i.clamp(max=B - 1)
    pos = lens.long()[i_] + t - start[i_]
    live = (i < B) & served[i_]
    page = table[i_, (pos // PAGE).clamp(max=W - 1)].long()
    slot_map = torch.where(live, page * PAGE + pos % PAGE, -1)
    positions = torch.where(live, pos, -1).int()
    taken = torch.where(served, need, 0).sum()
    counts = torch.stack([start[-1], taken, (~served).sum(), begin.long()[0] + taken]).int()
    return slot_map, positions, start.int(), torch.where(served, lens + new, lens), counts


def _run_append(s):
    if own:
        from paper_2609_37626_b200 import binding
        binding.splash_kv8_append(s["k"], s["v"], s["slot_map"], s["k_pool"], s["v_pool"], s["k_scales"], s["v_scales"])
    else:
        for x, pool, scales in ((s["k"], s["k_pool"], s["k_scales"]), (s["v"], s["v_pool"], s["v_scales"])):
            _plain_append(x.float(), s["slot_map"], s["first"], pool, scales)
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "k_scales": s["k_scales"], "v_scales": s["v_scales"]}


def _power(most):
    """The smallest power of two whose 448-fold is not below `most`."""
    m, e = torch.frexp(most)                   # most = m 2^e, m in [1/2, 1); 448 = 7/8 * 2^9
    return torch.where(most > 0, torch.exp2((e - 9 + (m > 0.875)).float()), 0.0).clamp(min=FLOOR)


def _plain_append(x, slot, first, pool, scales):
    page, row = slot // PAGE, slot % PAGE
    most = torch.zeros_like(scales).index_reduce_(0, page, x.abs().amax(-1), "amax")
    begin = torch.full((pool.shape[0],), PAGE, device=x.device).index_reduce_(0, page, row, "amin")
    old = torch.where(begin[:, None] == 0, 0.0, scales)
    need = _power(most)
    grown = torch.where((begin[:, None] < PAGE) & ~(old >= need), need, scales)
    # a page that was begun earlier is the first page of some request's new tokens: its older rows move to the new scale
    p = page[first]
    before = torch.arange(PAGE, device=x.device)[None, None, :, None] < row[first][:, None, None, None]
    kept = pool.view(torch.uint8)[p].view(E4M3).float() * scales[p][:, :, None, None]
    moved = (kept / grown[p][:, :, None, None]).clamp(-448, 448).to(E4M3)
    moves = before & (grown[p] != scales[p])[:, :, None, None]
    raw = pool.view(torch.uint8)
    raw[p] = torch.where(moves, moved.view(torch.uint8), raw[p])
    raw[page, :, row] = (x / grown[page][:, :, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
    scales.copy_(grown)


def _run_attention(s):
    if own:
        from paper_2609_37626_b200 import binding
        out, lse = binding.splash_kv8_attention(s["q"], s["k_pool"], s["v_pool"], s["k_scales"], s["v_scales"], s["block_table"], s["seq_lens"],
                                                softmax_scale=s["scale"], q_start=s["q_start"], max_q_rows=s["max_rows"])
    else:
        out, lse = _plain_attention(s["q"], s["k_pool"], s["v_pool"], s["k_scales"], s["v_scales"], s["block_table"], s["seq_lens"], s["scale"], s["q_start"],
                                    s["max_rows"])
    return {"out": out, "lse": lse}


def _dense(pool, scales, table, valid):
    """[B][heads][W * 64][D] in 32 bits, zeros where there is no token."""
    at = table.long().clamp(min=0)
    x = pool.view(torch.uint8)[at].view(E4M3).float() * scales[at][..., None, None]             # [B][W][heads][64][D]
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)
    return torch.where(valid[:, None, :, None], x, 0.0)


def _plain_attention(q, k_pool, v_pool, k_scales, v_scales, table, lens, scale, q_start, R):
    B, W = table.shape
    T, H, D = q.shape
    kv = k_pool.shape[1]
    dev = q.device
    if q_start is None:
        q_start = torch.arange(B + 1, device=dev)
    start, rows = q_start.long()[:-1], q_start.long()[1:] - q_start.long()[:-1]
    r = torch.arange(R, device=dev)
    x = q[(start[:, None] + r).clamp(max=T - 1)].float()                                        # [B][R][H][D]
    x = x.view(B, R, kv, H // kv, D).permute(0, 2, 3, 1, 4).reshape(B, kv, H // kv * R, D) * scale
    t = torch.arange(W * PAGE, device=dev)
    valid = t[None] < lens[:, None]
    logits = torch.matmul(x, _dense(k_pool, k_scales, table, valid).transpose(-1, -2)).view(B, kv, H // kv, R, W * PAGE)
    last = lens.long()[:, None] - rows[:, None] + r                                             # the row's own position
    logits = logits.masked_fill((t[None, None] > last[:, :, None])[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = torch.exp(logits - top)
    del logits
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, kv, H // kv * R, W * PAGE), _dense(v_pool, v_scales, table, valid)).view(B, kv, H // kv, R, D)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, R, H, D)
    lse = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(B, R, H)
    flat = torch.arange(T, device=dev)
    i = torch.searchsorted(q_start.long(), flat, right=True) - 1
    return out[i, flat - start[i]].to(q.dtype), lse[i, flat - start[i]]


# ---- the same from the definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"slots": _exact_slots, "append": _exact_append, "attention": _exact_attention}[case["op"]](s)


def _exact_slots(s):
    table, lens, new, free = (s[k].cpu().numpy().astype(np.int64) for k in ("block_table", "seq_lens", "new_lens", "free_pages"))
    B, W = table.shape
    at, left, taken, refused, end = 0, True, int(s["free_begin"][0]), 0, taken_from(s)
    slot_map, positions = np.full(s["num_slots"], -1, np.int64), np.full(s["num_slots"], -1, np.int32)
    q_start, after = [0], lens.copy()
    for i in range(B):
        q_start.append(at + int(new[i]))
        first, last = _pages(int(lens[i])), _pages(int(lens[i] + new[i]))
        need = last - first
        if last > W or q_start[-1] > s["num_slots"] or (need > 0 and not (left and taken + need <= len(free))):
            refused += 1
            if need > 0 and last <= W and q_start[-1] <= s["num_slots"]:
                left = False
        else:
            table[i, first:last] = free[taken:taken + need]
            taken += need
            after[i] = lens[i] + new[i]
            for j in range(int(new[i])):
                t = int(lens[i]) + j
                positions[at + j], slot_map[at + j] = t, table[i, t // PAGE] * PAGE + t % PAGE
        at = q_start[-1]
    whole = lambda x, t: torch.tensor(np.asarray(x), dtype=t)     # noqa: E731
    return {"block_table": whole(table, torch.int32), "slot_map": whole(slot_map, torch.int64), "positions": whole(positions, torch.int32),
            "q_start": whole(q_start, torch.int32), "new_seq_lens": whole(after, torch.int32), "counts": whole([at, taken - end, refused, taken], torch.int32)}


def taken_from(s):
    return int(s["free_begin"][0])


def _grid(x):
    """To the nearest value of e4m3, ties to the even one, in 64 bits."""
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))).clamp(min=-6) - 3)
    return torch.sign(x) * (torch.round(a / step) * step).clamp(max=448.0)


def _exact_append(s):
    out = {}
    slot = s["slot_map"].cpu().numpy()
    cut = [0] + [j for j in range(1, len(slot)) if slot[j] != slot[j - 1] + 1 or slot[j] % PAGE == 0] + [len(slot)]
    for name in ("k", "v"):
        x, pool, scales = s[name].double(), s[name + "_pool"].double(), s[name + "_scales"].double()
        for a, b in zip(cut, cut[1:]):
            p, r = int(slot[a]) // PAGE, int(slot[a]) % PAGE
            most = x[a:b].abs().amax(dim=(0, 2))
            need = torch.exp2(torch.ceil(torch.log2((most / 448).clamp(min=FLOOR))))
            old = scales[p].clone()
            scale = torch.maximum(old, need) if r else need
            kept = pool[p, :, :r]
            pool[p, :, :r] = torch.where((scale != old)[:, None, None], _grid(kept * (old / scale)[:, None, None]), kept)
            pool[p, :, r:r + b - a] = _grid(x[a:b] / scale[None, :, None]).transpose(0, 1)
            scales[p] = scale
        out[name + "_pool"], out[name + "_scales"] = pool, scales
    return out


def _exact_attention(s):
    lens = s["seq_lens"].tolist()
    ends = s["q_start"].tolist() if s["q_start"] is not None else list(range(len(lens) + 1))
    T, H, D = s["q"].shape
    kv = s["k_pool"].shape[1]
    out, lse = torch.empty((T, H, D), dtype=torch.float64, device="cuda"), torch.empty((T, H), dtype=torch.float64, device="cuda")
    for i, n in enumerate(lens):
        a, b = ends[i], ends[i + 1]
        pages = s["block_table"][i, :_pages(n)].long()
        k, v = ((s[x + "_pool"].view(torch.uint8)[pages].view(E4M3).double() * s[x + "_scales"][pages].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :n]
                for x in "kv")                                                                  # [kv][n][D]
        for h in range(H):
            logits = s["q"][a:b, h].double() @ k[h // (H // kv)].T * s["scale"]
            hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - (b - a), n, device="cuda")[:, None]
            logits = logits.masked_fill(hidden, -math.inf)
            lse[a:b, h] = torch.logsumexp(logits, -1)
            out[a:b, h] = torch.softmax(logits, -1) @ v[h // (H // kv)]
    return {"out": out, "lse": lse}
