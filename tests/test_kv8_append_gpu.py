"""Writing keys and values into the e4m3 cache against the definition in 64 bits.  A scale is a power of two and a code is rounded once, so
both are equal, not near."""
import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def slots_for(g, lens, new, P):
    """Slots of each request's new tokens behind its old ones, on random pages."""
    order, at, out = g.permutation(P), 0, []
    for a, b in zip(lens, new):
        pages = order[at:at + -(-(a + b) // 64) + 1]
        at += len(pages)
        t = np.arange(a, a + b)
        out.append(pages[t // 64].astype(np.int64) * 64 + t % 64)
    assert at <= P
    return np.concatenate(out) if out else np.zeros(0, np.int64)


def pool(g, P, heads, D, odd_scales=False):
    codes = g.integers(0, 256, (P, heads, 64, D)).astype(np.uint8)
    scales = np.exp2(g.integers(-12, 3, (P, heads))).astype(np.float32)
    if odd_scales:
        scales = (scales * g.uniform(1.0, 2.0, scales.shape)).astype(np.float32)
    return codes, scales


def inputs(g, n, heads, D, dtype):
    x = g.normal(size=(n, heads, D)) * np.exp2(g.integers(-6, 6, (n, heads, 1)))
    return torch.from_numpy(x).to(TYPES[dtype])


def run_and_compare(x, slot_map, pools, scales, view=None):
    P = pools[0].shape[0]
    cu = [torch.from_numpy(p).cuda() for p in pools]
    cs = [torch.from_numpy(s).cuda() for s in scales]
    args = [t.cuda() for t in x] if view is None else view(x)
    B.splash_kv8_append(*args, torch.from_numpy(slot_map).cuda(), *cu, *cs)
    torch.cuda.synchronize()
    for k in range(2):
        ref_v, ref_s = _kv8.append(x[k].double().numpy(), slot_map, _kv8.E4M3[pools[k]], scales[k])
        got_v, got_s = _kv8.E4M3[cu[k].cpu().numpy()], cs[k].cpu().numpy()
        assert np.array_equal(got_s.astype(np.float64), ref_s, equal_nan=True), "scales"
        assert np.array_equal(got_v, ref_v, equal_nan=True), f"codes: {(~np.isclose(got_v, ref_v, rtol=0, atol=0, equal_nan=True)).sum()} differ"
        untouched = np.ones(P, bool)
        untouched[[p for _, _, p, _ in _kv8.runs(slot_map, P)]] = False
        assert np.array_equal(cu[k].cpu().numpy()[untouched], pools[k][untouched])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,new", [([0], [1]), ([63], [1]), ([64], [64]), ([5, 0, 63, 64, 127, 200], [1, 1, 1, 1, 1, 1]), ([10, 0, 61, 1], [200, 64, 7, 130]),
                                      (list(range(70)), [1] * 70), ([3, 50, 0], [1, 300, 129])])
def test_runs(D, dtype, lens, new):
    g = np.random.default_rng([len(lens), sum(new), D])
    P, heads = sum(-(-(a + b) // 64) + 1 for a, b in zip(lens, new)) + 4, 3
    made = [pool(g, P, heads, D) for _ in range(2)]
    run_and_compare([inputs(g, sum(new), heads, D, dtype) for _ in range(2)], slots_for(g, lens, new, P), [m[0] for m in made], [m[1] for m in made])


@pytest.mark.parametrize("heads,total", [(1, 3000), (8, 2900), (2, 12000)])
def test_every_width_of_window(heads, total):
    # windows of 8 tokens and of 64, cut anywhere: prompts and single tokens mixed
    g = np.random.default_rng(heads)
    new = []
    while sum(new) < total:
        new += [int(g.integers(1, 400))] + [1] * int(g.integers(0, 60))
    lens = [int(v) for v in g.integers(0, 100, len(new))]
    P = sum(-(-(a + b) // 64) + 1 for a, b in zip(lens, new)) + 4
    made = [pool(g, P, heads, 64) for _ in range(2)]
    run_and_compare([inputs(g, sum(new), heads, 64, "bf16") for _ in range(2)], slots_for(g, lens, new, P), [m[0] for m in made], [m[1] for m in made])


def test_rows_without_a_place_are_skipped():
    g = np.random.default_rng(2)
    lens, new = [5, 60, 0, 7], [90, 70, 3, 1]
    P = 20
    slot_map = slots_for(g, lens, new, P)
    slot_map[20:50] = -1
    slot_map[100:103] = 64 * P + 5
    slot_map[103] = np.iinfo(np.int64).min
    slot_map[104] = np.iinfo(np.int64).max
    slot_map = np.concatenate([slot_map, np.full(200, -1)])
    # what is left of a page must be one run: the rows in front of the gap that share a page with rows behind it go as well
    seen = {}
    for j, s in enumerate(slot_map):
        if 0 <= s < 64 * P:
            seen.setdefault(int(s) // 64, []).append(j)
    for js in seen.values():
        for a, b in zip(js, js[1:]):
            if b != a + 1:
                slot_map[js[0]:a + 1] = -1
    made = [pool(g, P, 2, 128) for _ in range(2)]
    run_and_compare([inputs(g, len(slot_map), 2, 128, "bf16") for _ in range(2)], slot_map, [m[0] for m in made], [m[1] for m in made])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_at_the_edges(dtype):
    # zeros, infinities, NaN, the largest and smallest values, scales that are no power of two or no number
    g = np.random.default_rng(3)
    lens, new, heads, D = [0, 10, 20, 30, 40, 63, 64 * 3], [70, 3, 64, 1, 100, 2, 1], 4, 64
    P = sum(-(-(a + b) // 64) + 1 for a, b in zip(lens, new)) + 2
    x = []
    for _ in range(2):
        t = inputs(g, sum(new), heads, D, dtype)
        big, tiny = (3e38, 1e-40) if dtype == "bf16" else (65504.0, 6e-8)
        t[:30, 0] = 0.0
        t[5, 1, 3], t[6, 1, 4], t[7, 1, 5] = float("inf"), float("-inf"), float("nan")
        t[40, 2, :] = big
        t[72, 1] = float("nan")
        t[74:140, 3] = tiny
        t[73, 0] = -big
        t[140:, 2] = 0.0
        x.append(t)
    made = [pool(g, P, heads, D, odd_scales=True) for _ in range(2)]
    made[0][1][::3, 1] = np.nan
    made[1][1][::4, 2] = 2.0 ** 90
    made[1][1][1::4, 2] = 0.0
    run_and_compare(x, slots_for(g, lens, new, P), [m[0] for m in made], [m[1] for m in made])


def test_keys_and_values_in_a_wider_row():
    # k and v as slices of one projection's rows, pools as a rank's heads of a pool that holds keys and values side by side
    g = np.random.default_rng(4)
    lens, new, heads, D = [5, 100, 0], [70, 1, 40], 2, 128
    P = 12
    x = [inputs(g, sum(new), heads, D, "bf16") for _ in range(2)]
    slot_map = slots_for(g, lens, new, P)
    row = torch.zeros((sum(new), 6 * D + heads * 2 * D + 8), dtype=torch.bfloat16, device="cuda")
    k, v = (row[:, 6 * D + i * heads * D:6 * D + (i + 1) * heads * D].view(sum(new), heads, D) for i in range(2))
    k.copy_(x[0]), v.copy_(x[1])
    both = torch.from_numpy(g.integers(0, 256, (P, 2, 5, 64, D)).astype(np.uint8)).cuda()
    scales = torch.from_numpy(np.exp2(g.integers(-12, 3, (P, 10))).astype(np.float32)).cuda()
    before, scales_before = both.cpu().numpy(), scales.cpu().numpy()
    parts = [both[:, i, 1:3].view(torch.float8_e4m3fn) for i in range(2)]
    scale_parts = [scales[:, 3:5], scales[:, 8:10]]
    B.splash_kv8_append(k, v, torch.from_numpy(slot_map).cuda(), *parts, *scale_parts)
    after, scales_after = both.cpu().numpy(), scales.cpu().numpy()
    for i, cols in enumerate((slice(3, 5), slice(8, 10))):
        ref_v, ref_s = _kv8.append(x[i].double().numpy(), slot_map, _kv8.E4M3[before[:, i, 1:3]], scales_before[:, cols])
        assert np.array_equal(_kv8.E4M3[after[:, i, 1:3]], ref_v, equal_nan=True) and np.array_equal(scales_after[:, cols], ref_s)
    assert np.array_equal(after[:, :, [0, 3, 4]], before[:, :, [0, 3, 4]])
    assert np.array_equal(scales_after[:, [0, 1, 2, 5, 6, 7]], scales_before[:, [0, 1, 2, 5, 6, 7]])


def test_the_same_context_in_one_call_or_token_by_token():
    # scales are powers of two: but for values below the normal range, cutting a context into calls changes nothing
    g = np.random.default_rng(6)
    n, heads, D = 150, 2, 64
    x = torch.from_numpy(g.uniform(0.5, 1.0, (n, heads, D)) * np.sign(g.normal(size=(n, heads, D))) * np.exp2(np.arange(n) // 40)[:, None, None]).to(torch.bfloat16).cuda()
    slot_map = torch.arange(n, device="cuda")
    got = []
    for cuts in ([n], [1] * n, [7, 60, 1, 40, 42]):
        pools = [torch.zeros((3, heads, 64, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.full((3, heads), float("nan"), device="cuda") for _ in range(2)]
        at = 0
        for c in cuts:
            B.splash_kv8_append(x[at:at + c], x[at:at + c], slot_map[at:at + c], *pools, *scales)
            at += c
        got.append((pools[0].cpu(), scales[0].cpu()))
        assert torch.equal(pools[0], pools[1])
    assert all(torch.equal(a, got[0][0]) and torch.equal(s, got[0][1]) for a, s in got)


def test_pages_behind_four_gigabytes():
    P, heads, D = 70000, 8, 128              # 4.6 GB of keys, and of values
    pools = [torch.empty((P, heads, 64, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((P, heads), device="cuda") for _ in range(2)]
    g = np.random.default_rng(8)
    x = [inputs(g, 65, heads, D, "bf16") for _ in range(2)]
    slot_map = np.arange(64 * (P - 2), 64 * (P - 2) + 65)
    B.splash_kv8_append(x[0].cuda(), x[1].cuda(), torch.from_numpy(slot_map).cuda(), *pools, *scales)
    for k in range(2):
        ref_v, ref_s = _kv8.append(x[k].double().numpy(), slot_map - 64 * (P - 2), np.zeros((2, heads, 64, D)), np.ones((2, heads)))
        got = _kv8.E4M3[pools[k][P - 2:].cpu().numpy()]
        assert np.array_equal(got[0], ref_v[0]) and np.array_equal(got[1, :, 0], ref_v[1, :, 0]) and np.array_equal(scales[k][P - 2:].cpu().numpy(), ref_s)
