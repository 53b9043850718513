"""Appends in which a block takes several heads of its window one after the other: with that many windows, or that many heads, that there are
eight blocks an SM.  Pages begun earlier, scales that move for some heads and stay for others, values that are not finite in some heads: what one
head leaves behind in the block must not reach the next but one.  Equal to the definition in 64 bits."""
import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def folded(rows, heads, sms):
    """Heads that a block takes, by the launcher's rule: windows of 64 tokens (of 16 up to 512 rows), groups of heads halved while eight blocks an SM remain."""
    blocks, groups = -(-rows // (16 if rows <= 512 else 64)), heads
    while groups > 1 and blocks * ((groups + 1) // 2) * 2 >= 8 * sms:
        groups = (groups + 1) // 2
    return -(-heads // groups)


def batch(g, total):
    """Old and new tokens of requests, and slots of the new ones on random pages: prompts, chunks and single tokens that begin anywhere in a page."""
    new = []
    while sum(new) < total:
        new += [int(g.integers(1, 300))] + [1] * int(g.integers(0, 20)) + [64, 65][:int(g.integers(0, 3))]
    while sum(new) > total:
        last = new.pop()
        new += [last - (sum(new) + last - total)] if sum(new) < total else []
    lens = [int(v) for v in g.integers(0, 130, len(new))]
    pages = [-(-(a + b) // 64) for a, b in zip(lens, new)]
    P = sum(pages) + 3
    order, at, out = g.permutation(P), 0, []
    for a, b, n in zip(lens, new, pages):
        t = np.arange(a, a + b)
        out.append(order[at:at + n][t // 64].astype(np.int64) * 64 + t % 64)
        at += n
    return np.concatenate(out), P


def plain(x, slot_map, values, scales):
    """The definition, all heads of a run at once: values [P][heads][64][D] of the codes, scales [P][heads], both changed in place."""
    for a, b, p, r in _kv8.runs(slot_map, len(values)):
        rows = np.where(np.isfinite(x[a:b]), x[a:b], np.nan)
        most = np.nan_to_num(np.abs(rows)).max(axis=(0, 2))
        m, e = np.frexp(most)                                    # most = m 2^e, 448 = 7/8 2^9
        need = np.maximum(np.where(most > 0, np.ldexp(1.0, e - 9 + (m > 0.875)), 0.0), 2.0 ** -100)
        old = scales[p].copy()
        s = np.where((old >= need) & (r > 0), old, need)
        moves = (s != old) & (r > 0)
        values[p, moves, :r] = _kv8.to_grid((values[p, moves, :r] * old[moves, None, None]).astype(np.float32).astype(np.float64) / s[moves, None, None])
        q = rows / s[None, :, None]
        exact = np.frexp(s)[0] == 0.5
        q = np.where(exact[None, :, None], q, q.astype(np.float32).astype(np.float64))
        values[p, :, r:r + b - a] = _kv8.to_grid(q).transpose(1, 0, 2)
        scales[p] = s


# (rows, heads): many windows of a few heads; many heads of few windows; windows of 16 tokens; odd numbers of heads, whose last group is shorter
@pytest.mark.parametrize("dtype,D,rows,heads", [("bf16", 64, 20_000, 8), ("fp16", 64, 20_000, 4), ("bf16", 128, 2900, 33), ("fp16", 128, 2900, 64), ("bf16", 64, 500, 130),
                                                ("fp16", 128, 300, 97), ("bf16", 128, 19_000, 5)])
def test_blocks_that_take_several_heads(dtype, D, rows, heads):
    assert folded(rows, heads, torch.cuda.get_device_properties(0).multi_processor_count) >= 2
    g = np.random.default_rng([rows, heads, D])
    slot_map, P = batch(g, rows)
    codes, scales, xs = [], [], []
    for _ in range(2):
        c = g.integers(0, 256, (P, heads, 64, D), dtype=np.uint8)
        s = np.exp2(g.integers(-12, 3, (P, heads))).astype(np.float32)
        s[:, 1::3] *= 1.3                                            # (no powers of two)
        s[g.random(s.shape) < 0.03] = np.nan
        s[g.random(s.shape) < 0.03] = 0.0
        s[g.random(s.shape) < 0.03] = 2.0 ** 40                      # stays
        x = torch.from_numpy(g.normal(size=(rows, heads, D)).astype(np.float32) * np.exp2(g.integers(-8, 6, (rows, heads, 1))).astype(np.float32)).to(TYPES[dtype])
        for value, share in ((float("nan"), 0.004), (float("inf"), 0.004), (float("-inf"), 0.004)):
            x[..., int(g.integers(D))][torch.from_numpy(g.random((rows, heads)) < share) & (torch.arange(heads) % 2 == 1)] = value       # (odd heads alone)
        x[g.random(rows) < 0.05, heads // 2] = 0.0
        codes.append(c), scales.append(s), xs.append(x)
    cu, cs = [torch.from_numpy(c).cuda() for c in codes], [torch.from_numpy(s).cuda() for s in scales]
    B.splash_kv8_append(xs[0].cuda(), xs[1].cuda(), torch.from_numpy(slot_map).cuda(), *cu, *cs)
    torch.cuda.synchronize()
    touched = np.zeros(P, bool)
    touched[[p for _, _, p, _ in _kv8.runs(slot_map, P)]] = True
    for k in range(2):
        got = cu[k].cpu().numpy()
        assert np.array_equal(got[~touched], codes[k][~touched]) and np.array_equal(cs[k].cpu().numpy()[~touched], scales[k][~touched], equal_nan=True)
        for h0 in range(0, heads, 16):                               # (16 heads at a time: 64-bit values of all of them are gigabytes)
            part = slice(h0, h0 + 16)
            values, s = _kv8.E4M3[codes[k][:, part]], scales[k][:, part].astype(np.float64)
            plain(xs[k][:, part].double().numpy(), slot_map, values, s)
            assert np.array_equal(cs[k][:, part].cpu().numpy().astype(np.float64), s, equal_nan=True), f"scales of the heads from {h0} on"
            assert np.array_equal(_kv8.E4M3[got[:, part]], values, equal_nan=True), f"codes of the heads from {h0} on"


@pytest.mark.parametrize("heads,total", [(1, 40), (3, 512), (8, 511)])
def test_windows_of_sixteen_tokens(heads, total):
    g = np.random.default_rng([heads, total])
    slot_map, P = batch(g, total)
    x = torch.from_numpy(g.normal(size=(total, heads, 64)) * np.exp2(g.integers(-8, 6, (total, heads, 1)))).to(torch.bfloat16)
    c, s = g.integers(0, 256, (P, heads, 64, 64), dtype=np.uint8), np.exp2(g.integers(-12, 3, (P, heads))).astype(np.float32)
    cu, cs = [torch.from_numpy(c).cuda() for _ in range(2)], [torch.from_numpy(s).cuda() for _ in range(2)]
    B.splash_kv8_append(x.cuda(), x.cuda(), torch.from_numpy(slot_map).cuda(), *cu, *cs)
    values, ref_s = _kv8.E4M3[c], s.astype(np.float64)
    plain(x.double().numpy(), slot_map, values, ref_s)
    for k in range(2):
        assert np.array_equal(cs[k].cpu().numpy(), ref_s) and np.array_equal(_kv8.E4M3[cu[k].cpu().numpy()], values, equal_nan=True)
