"""Attention over the e4m3 cache of keys and values against the definition in 64 bits, within bounds that follow from its roundings."""
import math

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}


def queries(seed, T, H, D, dtype, size=1.0):
    return (torch.from_numpy(np.random.default_rng(seed).normal(size=(T, H, D))) * size).to(TYPES[dtype])


def attend(cache, q, rows, dtype="bf16", scale=None, kv=None, out_dtype=None, width=None, **kw):
    """One call and its comparison; rows: None (one each) or the number of each request's rows."""
    scale = 1.0 / math.sqrt(cache.D) if scale is None else scale
    tensors = cache.cuda()
    q_start = None if rows is None else np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    if q_start is not None:
        kw.setdefault("max_q_rows", max(max(rows), 1))
        kw["q_start"] = torch.from_numpy(q_start).cuda()
    if kv is not None:
        kw["kv_begin"], kw["kv_end"] = (None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda") for a in kv)
    if out_dtype == "fp32":
        kw["out"] = torch.full(q.shape, 7.0, device="cuda")
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    out, lse = B.splash_kv8_attention(q.cuda() if q.device.type == "cpu" else q, *tensors, softmax_scale=scale, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert B.splash_workspace_status(ws)[0] == 0
    begin, end = kv if kv is not None else (None, None)
    ref = _kv8.attention(cache, q.double().cpu().numpy(), q_start, scale, begin, end, HALF_STEP[out_dtype or dtype])
    _kv8.check((out.double().cpu().numpy(), lse.cpu().numpy()), ref)
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8, 16, 17, 32, 40])
def test_one_row(D, group, dtype):
    lens = [0, 1, 17, 64, 65, 200, 1000, 128, 2]
    cache = _kv8.Cache([D, group], lens, 2, D)
    attend(cache, queries(group, len(lens), 2 * group, D, dtype), None, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group,rows", [(1, [3, 1, 0, 8, 5, 2]), (4, [8, 8, 8, 8, 8, 8]), (5, [2, 7, 1, 1, 3, 8]), (8, [3, 0, 4, 2, 1, 6])])
def test_few_rows(D, group, rows):
    lens = [64, 1, 5, 300, 700, 9]
    cache = _kv8.Cache([D, group, 5], lens, 3, D)
    attend(cache, queries(7, sum(rows), 3 * group, D, "fp16"), rows, "fp16")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group,rows,lens", [(1, [65, 130, 257], [65, 500, 300]), (4, [100, 1, 33, 16, 17], [400, 90, 33, 80, 17]), (7, [61, 200], [700, 200]), (1, [1000], [1000]),
                                             (32, [9, 3], [100, 70]), (3, [128, 43], [129, 64 * 3])])
def test_chunks(D, dtype, group, rows, lens):
    cache = _kv8.Cache([D, group, 6], lens, 2, D)
    attend(cache, queries(8, sum(rows), 2 * group, D, dtype), rows, dtype)


def test_rows_in_front_of_the_sequence_are_empty():
    # more rows than tokens: the first ones sit at negative positions
    for rows in ([5, 8, 2], [200, 8, 70]):
        cache = _kv8.Cache(1, [3, 0, 64], 1, 128)
        attend(cache, queries(9, sum(rows), 4, 128, "bf16"), rows)


def test_contexts_that_are_cut_and_joined():
    for D, lens, H in ((128, [20000, 10, 3000], 4), (64, [30000], 2), (128, [9000] * 3, 40)):
        cache = _kv8.Cache(D, lens, 1 if H > 4 else 2, D)
        attend(cache, queries(10, len(lens), H, D, "bf16"), None)


def test_many_short_requests():
    g = np.random.default_rng(11)
    lens = [int(v) for v in g.integers(0, 130, 700)]
    cache = _kv8.Cache(11, lens, 1, 64)
    attend(cache, queries(11, 700, 4, 64, "bf16"), None)


@pytest.mark.parametrize("rows", [None, [4, 1, 8, 3, 2], [40, 100, 70, 3, 200]])
def test_ranges(rows):
    lens = [500, 130, 700, 64, 300]
    begin, end = [64, 3, 129, -5, 299], [500, 7, 650, 1000, 100]
    cache = _kv8.Cache(12, lens, 2, 128)
    T = 5 if rows is None else sum(rows)
    attend(cache, queries(12, T, 6, 128, "bf16"), rows, kv=(begin, end))
    attend(cache, queries(12, T, 6, 128, "bf16"), rows, kv=(None, end), out_dtype="fp32")
    attend(cache, queries(12, T, 6, 128, "bf16"), rows, kv=(begin, None), out_dtype="fp32")


@pytest.mark.parametrize("rows", [None, [20, 100]])
def test_ranges_merged_give_the_whole(rows):
    lens = [1500, 800]
    cache = _kv8.Cache(13, lens, 2, 64)
    T = 2 if rows is None else sum(rows)
    q = queries(13, T, 8, 64, "bf16")
    outs, lses = [], []
    for a, b in ((0, 100), (100, 777), (777, 5000)):
        o, l = attend(cache, q, rows, kv=([a] * 2, [b] * 2), out_dtype="fp32")
        outs.append(o.reshape(-1, 64)), lses.append(l.reshape(-1))
    out, lse = B.splash_lse_merge(torch.stack(outs), torch.stack(lses))
    q_start = None if rows is None else np.concatenate([[0], np.cumsum(rows)])
    ref = _kv8.attention(cache, q.double().numpy(), q_start, 0.125, out_eps=2.0 ** -20)
    _kv8.check((out.double().cpu().numpy().reshape(T, 8, 64), lse.cpu().numpy().reshape(T, 8)), ref)


def test_a_table_narrower_than_the_context():
    cache = _kv8.Cache(14, [400, 100], 1, 128)
    cache.table = np.ascontiguousarray(cache.table[:, :3])
    attend(cache, queries(14, 2, 4, 128, "bf16"), None)


def test_page_ids_outside_the_pool_read_as_zeros():
    cache = _kv8.Cache(15, [300, 200], 2, 128)
    cache.table[0, 1], cache.table[0, 3], cache.table[1, 0] = -1, cache.P, 2 ** 30
    attend(cache, queries(15, 2, 8, 128, "bf16"), None)
    attend(cache, queries(15, 160, 8, 128, "bf16"), [100, 60])


@pytest.mark.parametrize("rows", [None, [5, 2], [90, 70]])
def test_strides_and_rows_of_nobody(rows):
    # q as the first heads of a projection's rows, a wider out and lse, rows in front of and behind the batch
    lens, H, D = [200, 130], 6, 128
    cache = _kv8.Cache(16, lens, 2, D)
    T = 2 if rows is None else sum(rows)
    q = queries(16, T, H, D, "bf16")
    wide = torch.full((T + 5, H + 4, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full((T + 5, H + 1, D), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((T + 5, H + 9), 3.0, device="cuda")
    tensors = cache.cuda()
    table = torch.full((2, cache.table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    table[:, 1:-2] = tensors[4]
    if rows is None:
        wide[:T, 1:1 + H] = q.cuda()
        q_start, sub, kw = None, slice(0, T), {}
    else:
        wide[2:2 + T, 1:1 + H] = q.cuda()
        q_start, sub = np.concatenate([[2], 2 + np.cumsum(rows)]).astype(np.int32), slice(0, T + 5)
        kw = dict(q_start=torch.from_numpy(q_start).cuda(), max_q_rows=max(rows))
    B.splash_kv8_attention(wide[sub, 1:1 + H], *tensors[:4], table[:, 1:-2], tensors[5], softmax_scale=0.1, out=out[sub, :H], lse=lse[sub, 2:2 + H], **kw)
    first = 0 if rows is None else 2
    ref = _kv8.attention(cache, q.double().numpy(), None if rows is None else q_start - 2, 0.1, out_eps=2.0 ** -8)
    _kv8.check((out[first:first + T, :H].double().cpu().numpy(), lse[first:first + T, 2:2 + H].cpu().numpy()), ref)
    assert (out[:, H:] == 3).all() and (lse[:, :2] == 3).all() and (lse[:, 2 + H:] == 3).all()
    assert (out[:first] == 3).all() and (out[first + T:] == 3).all() and (lse[first + T:] == 3).all() and (lse[:first] == 3).all()


def test_more_rows_than_announced_are_left_alone():
    cache = _kv8.Cache(17, [300], 1, 64)
    q = queries(17, 100, 2, 64, "bf16").cuda()
    for most in (3, 90):
        out, lse = torch.full((100, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((100, 2), 9.0, device="cuda")
        B.splash_kv8_attention(q, *cache.cuda(), softmax_scale=0.1, q_start=torch.tensor([0, 100], dtype=torch.int32, device="cuda"), max_q_rows=most, out=out, lse=lse)
        ref = _kv8.attention(cache, q.double().cpu().numpy(), [0, 100], 0.1, out_eps=2.0 ** -8)
        _kv8.check((out[:most].double().cpu().numpy(), lse[:most].cpu().numpy()), [r[:most] for r in ref])
        assert (out[most:] == 9).all() and (lse[most:] == 9).all()


def test_sizes_of_queries_and_scales():
    # queries far outside fp16's range, value scales that differ by 2^20 between pages, logits in the hundreds
    lens = [700, 100]
    for size, scale, exps in ((1e30, 1e-31, (-9, -5)), (1e-30, 1e29, (-9, -5)), (1.0, 0.1, (-18, 2)), (40.0, 0.5, (-6, -5))):
        cache = _kv8.Cache(18, lens, 2, 128, scale_exp=exps)
        attend(cache, queries(18, 2, 8, 128, "bf16", size), None, scale=scale)
        attend(cache, queries(18, 130, 8, 128, "bf16", size), [90, 40], scale=scale)


def test_zero_queries_and_pages_of_zeros():
    cache = _kv8.Cache(19, [300, 70], 2, 128)
    for x in range(2):
        cache.codes[x][cache.table[0, 1]] = 0
        cache.scales[x][cache.table[0, 1]] = 2.0 ** -100
        cache.codes[x][cache.table[1, :2]] = 0
        cache.scales[x][cache.table[1, :2]] = 0.0
    q = queries(19, 2, 4, 128, "bf16")
    q[0, 1] = 0
    attend(cache, q, None)
    attend(cache, queries(19, 150, 4, 128, "bf16"), [100, 50])


@pytest.mark.parametrize("rows", [[4, 3], [150, 70]])
@pytest.mark.parametrize("which", ["key", "value", "key scale", "value scale", "query"])
def test_nan_stays_with_the_rows_that_see_it(rows, which):
    lens, D = [300, 200], 128
    cache = _kv8.Cache(20, lens, 2, D)
    q = queries(20, sum(rows), 4, D, "bf16")
    clean = [t.float().cpu().numpy() for t in attend(cache, q, rows)]
    t = lens[0] - 2                                     # the token of the last row but one of request 0
    page, r = cache.table[0, t // 64], t % 64
    sees = np.zeros((sum(rows), 4), bool)
    if which == "query":
        q[1, 2, 5] = float("nan")
        sees[1, 2] = True
    elif "scale" in which:                              # a whole page of one head
        cache.scales[which.startswith("value")][page, 1] = np.nan
        for k in range(rows[0]):
            sees[k, 2:] = lens[0] - rows[0] + k >= t // 64 * 64
    else:
        cache.codes[which == "value"][page, 1, r, 7] = 0x7F
        sees[rows[0] - 2:rows[0], 2:] = True
    kw = dict(softmax_scale=1 / math.sqrt(D), q_start=torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32, device="cuda"), max_q_rows=max(rows))
    out, lse = (x.float().cpu().numpy() for x in B.splash_kv8_attention(q.cuda(), *cache.cuda(), **kw))
    assert np.array_equal(lse[~sees], clean[1][~sees]) or which == "key scale" or np.allclose(lse[~sees], clean[1][~sees], rtol=0, atol=1e-5)
    assert np.isfinite(out[~sees]).all() and np.allclose(out[~sees], clean[0][~sees], rtol=2.0 ** -7, atol=2.0 ** -9 * np.abs(clean[0]).max())
    if which == "value":
        assert np.isnan(out[sees][:, 7]).all() and np.isfinite(np.delete(out[sees], 7, 1)).all() and np.isfinite(lse[sees]).all()
    elif which == "value scale":
        assert np.isnan(out[sees]).all() and np.isfinite(lse[sees]).all()
    else:
        assert np.isnan(out[sees]).all() and np.isnan(lse[sees]).all()


def test_one_answer_for_one_call():
    cache = _kv8.Cache(21, [5000, 300, 64, 1], 2, 128)
    for rows in (None, [300, 8, 1, 1]):
        T = 4 if rows is None else sum(rows)
        a = attend(cache, queries(21, T, 8, 128, "bf16"), rows)
        b = attend(cache, queries(21, T, 8, 128, "bf16"), rows)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_pages_behind_four_gigabytes():
    P, heads, D = 70000, 8, 128
    small = _kv8.Cache(22, [130], heads, D, spare=0)
    pools = [torch.empty((P, heads, 64, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((P, heads), device="cuda") for _ in range(2)]
    codes_k, codes_v, ks, vs, table, lens = small.cuda()
    for to, src in zip(pools + scales, (codes_k, codes_v, ks, vs)):
        to[P - 3:] = src
    for rows in (None, [100]):
        T = 1 if rows is None else 100
        q = queries(22, T, 16, D, "bf16")
        kw = {} if rows is None else dict(q_start=torch.tensor([0, 100], dtype=torch.int32, device="cuda"), max_q_rows=100)
        out, lse = B.splash_kv8_attention(q.cuda(), *pools, *scales, table + P - 3, lens, softmax_scale=0.1, **kw)
        _kv8.check((out.double().cpu().numpy(), lse.cpu().numpy()), _kv8.attention(small, q.double().numpy(), None if rows is None else [0, 100], 0.1, out_eps=2.0 ** -8))


def test_head_slices_of_shared_buffers():
    # a rank's key heads [1, 3) of 4, its query heads of a buffer with all of them
    cache = _kv8.Cache(23, [400, 90], 4, 64)
    q = queries(23, 2, 12, 64, "bf16")
    ck, cv, ks, vs, table, lens = cache.cuda()
    out, lse = torch.zeros((2, 12, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 12), device="cuda")
    for a, b in ((1, 3), (0, 1), (3, 4)):
        B.splash_kv8_attention(q.cuda()[:, 3 * a:3 * b], ck[:, a:b], cv[:, a:b], ks[:, a:b], vs[:, a:b], table, lens, softmax_scale=0.125, out=out[:, 3 * a:3 * b],
                               lse=lse[:, 3 * a:3 * b])
    _kv8.check((out.double().cpu().numpy(), lse.cpu().numpy()), _kv8.attention(cache, q.double().numpy(), None, 0.125, out_eps=2.0 ** -8))


@pytest.mark.parametrize("rows", [None, [70, 40]])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30])
def test_odd_softmax_scales(rows, scale):
    cache = _kv8.Cache(24, [200, 90], 2, 128)
    attend(cache, queries(24, 2 if rows is None else sum(rows), 8, 128, "bf16"), rows, scale=scale)


@pytest.mark.parametrize("rows", [None, [50, 90]])
def test_a_table_without_columns(rows):
    cache = _kv8.Cache(25, [200, 90], 2, 64)
    cache.table = np.zeros((2, 0), np.int32)
    out, lse = attend(cache, queries(25, 2 if rows is None else sum(rows), 4, 64, "fp16"), rows, "fp16")
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_requests_without_tokens_anywhere_on_the_line():
    # many empty requests between long ones: wherever the work is cut, their outputs are written where they belong
    for D, group in ((64, 1), (128, 4), (128, 16)):
        lens = [0, 0, 3000, 0, 1, 0, 0, 0, 2000] + [0] * 60 + [700, 0]
        cache = _kv8.Cache([26, D], lens, 1, D)
        attend(cache, queries(26, len(lens), group, D, "bf16"), None)


def test_many_key_heads_and_wide_groups():
    cache = _kv8.Cache(27, [130, 70], 33, 64)
    attend(cache, queries(27, 2, 33, 64, "bf16"), None)
    cache = _kv8.Cache(28, [300, 5], 1, 128)
    attend(cache, queries(28, 2, 128, 128, "bf16"), None)
    attend(cache, queries(28, 6, 200, 128, "fp16"), [4, 2], "fp16")


def test_chunks_cut_and_joined():
    # few tiles over long contexts: pages of one tile are spread over many workers
    for D, rows, lens, kv in ((128, [200], [20000], 1), (64, [40, 3], [30000, 9000], 2)):
        cache = _kv8.Cache([29, D], lens, kv, D)
        attend(cache, queries(29, sum(rows), 4 * kv, D, "bf16"), rows)


def test_a_batch_of_many_chunks():
    g = np.random.default_rng(30)
    rows = [int(v) for v in g.integers(0, 70, 90)]
    lens = [r + int(v) for r, v in zip(rows, g.integers(0, 300, 90))]
    cache = _kv8.Cache(30, lens, 1, 64)
    attend(cache, queries(30, sum(rows), 2, 64, "bf16"), rows)
