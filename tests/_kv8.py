"""Plain implementations, in 64 bits, of the operators around the 8-bit cache of keys and values, and inputs for their tests."""
import math

import numpy as np

PAGE = 64


def _table():
    """The values of the 256 e4m3 codes."""
    v = np.empty(256)
    for code in range(256):
        sign, e, m = (-1.0 if code & 0x80 else 1.0), code >> 3 & 15, code & 7
        v[code] = math.nan if e == 15 and m == 7 else sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return v


E4M3 = _table()


def to_grid(x):
    """The nearest e4m3 value, ties to even, clamped to 448; NaN stays NaN."""
    a = np.minimum(np.abs(x), 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    step = 2.0 ** (e - 3)
    return np.sign(x) * np.minimum(np.round(a / step) * step, 448.0)


def power_of_two_scale(most):
    """Smallest power of two s with most <= 448 s, at least 2^-100."""
    s = 2.0 ** -100
    return s if most <= 448 * s else 2.0 ** math.ceil(math.log2(most / 448.0))


# ---- places ----------------------------------------------------------------------------------------------------------------

def slots(table, lens, new, free, begin, num_slots):
    """(table, slot_map, positions, q_start, new_seq_lens, counts)"""
    table, W = table.copy(), table.shape[1]
    slot_map, positions = np.full(num_slots, -1, np.int64), np.full(num_slots, -1, np.int32)
    q_start, after = [0], []
    taken, refused, dry = 0, 0, False
    available = len(free) - begin if 0 <= begin < len(free) else 0
    for i in range(len(lens)):
        old, more = max(int(lens[i]), 0), max(int(new[i]), 0)
        at = q_start[-1]
        q_start.append(at + more)
        have, want = -(-old // PAGE), -(-(old + more) // PAGE)
        served = want <= W and at + more <= num_slots and old + more <= 2 ** 31 - 1
        if served and want > have:
            if dry or taken + want - have > available:
                served, dry = False, True
        if not served:
            refused += 1
            after.append(old)
            continue
        table[i, have:want] = free[begin + taken:begin + taken + want - have]
        taken += want - have
        after.append(old + more)
        for j in range(more):
            positions[at + j] = old + j
            slot_map[at + j] = PAGE * int(table[i, (old + j) // PAGE]) + (old + j) % PAGE
    return table, slot_map, positions, np.minimum(q_start, 2 ** 31 - 1).astype(np.int32), np.array(after, np.int32), np.array([min(q_start[-1], 2 ** 31 - 1), taken, refused, begin + taken], np.int32)


# ---- append ----------------------------------------------------------------------------------------------------------------

def runs(slot_map, num_pages):
    out, j, n = [], 0, len(slot_map)
    while j < n:
        s = int(slot_map[j])
        if s < 0 or s // PAGE >= num_pages:
            j += 1
            continue
        k = j + 1
        while k < n and int(slot_map[k]) == int(slot_map[k - 1]) + 1 and int(slot_map[k]) % PAGE:
            k += 1
        out.append((j, k, s // PAGE, s % PAGE))
        j = k
    return out


def append(x, slot_map, values, scales):
    """x [N][heads][D] float64; values [P][heads][64][D] the codes' values, scales [P][heads]: both are returned as they are after the call."""
    values, scales = values.copy(), scales.astype(np.float64)
    for a, b, p, r in runs(slot_map, values.shape[0]):
        for h in range(x.shape[1]):
            rows = x[a:b, h]
            finite = np.abs(rows[np.isfinite(rows)])
            need = power_of_two_scale(finite.max() if finite.size else 0.0)
            old = scales[p, h]
            s = old if r > 0 and old >= need else need
            if r > 0 and s != old:
                values[p, h, :r] = to_grid((values[p, h, :r] * old).astype(np.float32).astype(np.float64) / s)
            rows = np.where(np.isfinite(rows), rows, np.nan)
            q = rows / s
            if np.log2(s) != np.floor(np.log2(s)):
                q = q.astype(np.float32).astype(np.float64)
            values[p, h, r:r + b - a] = to_grid(q)
            scales[p, h] = s
    return values, scales


# ---- attention -------------------------------------------------------------------------------------------------------------

class Cache:
    """A random cache: codes [P][heads][64][D] and scales of keys and values, a block table, poison wherever no token is."""

    def __init__(self, seed, lens, heads, D, width=None, spare=3, scale_exp=(-9, -5)):
        g = np.random.default_rng(seed)
        pages = [-(-n // PAGE) for n in lens]
        P = sum(pages) + spare
        order = g.permutation(P)
        W = max(pages + [1]) if width is None else width
        self.table = np.full((len(lens), W), -7, np.int32)
        self.lens, self.heads, self.D, self.P = np.array(lens, np.int32), heads, D, P
        self.codes = [np.full((P, heads, PAGE, D), 0x7F, np.uint8) for _ in range(2)]
        self.scales = [np.full((P, heads), np.nan, np.float32) for _ in range(2)]
        at = 0
        for i, n in enumerate(lens):
            self.table[i, :pages[i]] = order[at:at + pages[i]]
            for j, p in enumerate(order[at:at + pages[i]]):
                m = min(PAGE, n - PAGE * j)
                for x in range(2):
                    c = g.integers(0, 256, (heads, m, D)).astype(np.uint8)
                    c[(c & 0x7F) == 0x7F] = 0x30
                    self.codes[x][p, :, :m] = c
                    self.scales[x][p] = np.exp2(g.integers(scale_exp[0], scale_exp[1] + 1, heads)) * g.choice([1.0, 1.3])
            at += pages[i]

    def dense(self, i, n=None):
        """Keys and values of request i, [heads][n][D] in 64 bits; pages outside the pool are zeros."""
        n = int(self.lens[i]) if n is None else n
        out = []
        for x in range(2):
            d = np.zeros((self.heads, n, self.D))
            for j in range(-(-n // PAGE)):
                p = int(self.table[i, j])
                m = min(PAGE, n - PAGE * j)
                if 0 <= p < self.P:
                    d[:, PAGE * j:PAGE * j + m] = E4M3[self.codes[x][p, :, :m]] * self.scales[x][p].astype(np.float64)[:, None, None]
            out.append(d)
        return out

    def cuda(self):
        import torch
        return [torch.from_numpy(a).cuda() for a in (*self.codes, *self.scales, self.table, self.lens)]


def attention(cache, q, q_start, scale, kv_begin=None, kv_end=None, out_eps=2.0 ** -9):
    """(out, lse, bound of out, bound of lse) of every row that belongs to a request, NaN elsewhere.

    The bounds: a softmax weight is rounded to fp16 (2^-11 relative, 2^-31 of the largest weight absolutely); a logit is summed in fp32 over D
    exact products (D / 2^23 of the sum of their sizes) and then subject to a few fp32 roundings; sums over n tokens in fp32 add n / 2^22 at most; the
    output is rounded once to its type, half a step `out_eps`: relative to the value, and in fp16 below 2^-14, where the values lie 2^-24 apart, 2^-25."""
    T, H, D = q.shape
    group = H // cache.heads
    out, lse = np.full((T, H, D), np.nan), np.full((T, H), np.nan)
    tol, tol_lse = np.zeros((T, H, D)), np.zeros((T, H))
    width = cache.table.shape[1] * PAGE
    for i, n in enumerate(cache.lens):
        a, b = (int(q_start[i]), int(q_start[i + 1])) if q_start is not None else (i, i + 1)
        n = int(n)
        keys, values = cache.dense(i, min(n, width))
        for t in range(a, b):
            lo = 0 if kv_begin is None else max(int(kv_begin[i]), 0)
            hi = min(n - (b - a) + (t - a) + 1, width)
            if kv_end is not None:
                hi = min(hi, int(kv_end[i]))
            for g in range(H):
                if hi <= lo:
                    out[t, g], lse[t, g] = 0.0, -np.inf
                    continue
                k, v = keys[g // group, lo:hi], values[g // group, lo:hi]
                x = k @ q[t, g] * scale
                m = x.max()
                p = np.exp(x - m)
                total = p.sum()
                out[t, g], lse[t, g] = p @ v / total, m + math.log(total)
                off = float((np.abs(k) @ np.abs(q[t, g])).max() * abs(scale)) * (D + 16) * 2.0 ** -23 + 2.0 ** -20
                spread = p @ np.abs(v) / total
                tol[t, g] = spread * (2.0 ** -11 + 2 * off + (hi - lo) * 2.0 ** -22) + (hi - lo) * 2.0 ** -31 * np.abs(v).max() / total + out_eps * np.abs(out[t, g]) + (2.0 ** -25 if out_eps == 2.0 ** -11 else 1e-30)
                tol_lse[t, g] = off + (hi - lo) * 2.0 ** -22 + 2.0 ** -21 + 2.0 ** -22 * abs(lse[t, g])
    return out, lse, tol, tol_lse


def check(got, ref):
    """got (out, lse) as float arrays against attention()'s answer; rows that it has NaN for are not looked at."""
    out, lse, tol, tol_lse = ref
    rows = ~np.isnan(lse[:, 0])
    o, l = got[0][rows].astype(np.float64), got[1][rows].astype(np.float64)
    empty = np.isneginf(lse[rows])
    assert np.isneginf(l[empty]).all() and (o[empty] == 0).all(), "an empty row"
    o, l, ro, rl, to, tl = o[~empty], l[~empty], out[rows][~empty], lse[rows][~empty], tol[rows][~empty], tol_lse[rows][~empty]
    assert np.isfinite(o).all() and np.isfinite(l).all(), "not finite"
    if o.size:
        assert (np.abs(l - rl) <= tl).all(), f"lse off by {np.abs(l - rl).max()}, {(np.abs(l - rl) / tl).max()} of the bound"
        assert (np.abs(o - ro) <= to).all(), f"out off by {(np.abs(o - ro) / to).max()} of the bound at {np.unravel_index((np.abs(o - ro) / to).argmax(), o.shape)}"
