"""The value scale of a page of which a row sees no token (those behind a causal row that later rows of its request see) may be anything: the
row's result is that of its own tokens."""
import math

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu


def attend(cache, q, rows):
    q_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
    got = B.splash_kv8_attention(q.cuda(), *cache.cuda(), softmax_scale=1 / math.sqrt(cache.D), q_start=torch.from_numpy(q_start).cuda(), max_q_rows=max(rows), out=out)
    return [t.double().cpu().numpy() for t in got], q_start


# rows of one request each, and its context: the last page (or two) is hidden from the first rows.  Few rows and many, whole contexts and such as are
# cut and joined, one tile of rows and several
CHUNKS = [([150], [200], 4), ([300, 70], [300, 75], 1), ([90], [9000], 2)]

FEW = [([4], [66], 4), ([8, 3, 5], [70, 129, 5001], 2), ([8], [68], 3), ([5], [29955], 1), ([4, 4], [65, 130], 8), ([2, 2, 2], [65, 641, 1], 8)]


def last_page_scaled(rows, lens, group, D, scale):
    heads = 2
    cache = _kv8.Cache([41, D, group], lens, heads, D)
    q = torch.from_numpy(np.random.default_rng(41).normal(size=(sum(rows), heads * group, D))).to(torch.float16)
    q_start = np.concatenate([[0], np.cumsum(rows)])
    ref = [a.copy() for a in _kv8.attention(cache, q.double().numpy(), q_start, 1 / math.sqrt(D), out_eps=2.0 ** -24)]
    blind = np.zeros(sum(rows), bool)                    # rows that see no token of their request's last page
    for i, n in enumerate(lens):
        first = (n - 1) // 64 * 64
        cache.scales[1][cache.table[i, first // 64]] = scale
        blind[q_start[i]:q_start[i + 1]] = n - rows[i] + np.arange(rows[i]) < first
    assert blind.any() and not blind.all()
    got, _ = attend(cache, q, rows)
    _kv8.check([a[blind] for a in got], [a[blind] for a in ref])
    return cache, q, q_start, got


@pytest.mark.parametrize("scale", [2.0 ** 60, 2.0 ** 115, -1e38, 3e38, np.inf, np.nan, 0.0, 1e-40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,lens,group", CHUNKS)
def test_chunks(rows, lens, group, D, scale):
    last_page_scaled(rows, lens, group, D, scale)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,lens,group", CHUNKS)
def test_rows_that_see_the_page_have_its_scale(rows, lens, group, D):
    # 2^100: what the other pages add to such a row is below its rounding
    cache, q, q_start, got = last_page_scaled(rows, lens, group, D, 2.0 ** 100)
    _kv8.check(got, _kv8.attention(cache, q.double().numpy(), q_start, 1 / math.sqrt(D), out_eps=2.0 ** -24))


@pytest.mark.parametrize("scale", [2.0 ** 60, 2.0 ** 115, -1e38, 3e38, np.inf, np.nan, 0.0, 1e-40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,lens,group", FEW)
def test_few_rows(rows, lens, group, D, scale):
    last_page_scaled(rows, lens, group, D, scale)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,lens,group", FEW)
def test_few_rows_that_see_the_page_have_its_scale(rows, lens, group, D):
    cache, q, q_start, got = last_page_scaled(rows, lens, group, D, 2.0 ** 100)
    _kv8.check(got, _kv8.attention(cache, q.double().numpy(), q_start, 1 / math.sqrt(D), out_eps=2.0 ** -24))


@pytest.mark.parametrize("scales", [(1e38, 3e38), (2.0 ** 53, 2.0 ** 113), (3e38, 1.0), (2.0 ** -3, 2.0 ** 126)])
@pytest.mark.parametrize("most", [40, 90])
def test_several_pages_behind_a_row(most, scales):
    # of 150 announced rows at the positions from 150 on the first `most` are computed: the last pages, from 192 and 256 on, are hidden from all or some of them
    cache = _kv8.Cache(42, [300], 1, 64)
    q = torch.from_numpy(np.random.default_rng(42).normal(size=(150, 1, 64))).to(torch.bfloat16)
    ref = [a.copy() for a in _kv8.attention(cache, q.double().numpy(), [0, 150], 0.125, out_eps=2.0 ** -24)]
    cache.scales[1][cache.table[0, 3]], cache.scales[1][cache.table[0, 4]] = scales
    out, lse = torch.empty((150, 1, 64), device="cuda"), torch.empty((150, 1), device="cuda")
    B.splash_kv8_attention(q.cuda(), *cache.cuda(), softmax_scale=0.125, q_start=torch.tensor([0, 150], dtype=torch.int32, device="cuda"), max_q_rows=most, out=out, lse=lse)
    blind = slice(0, 192 - 150 if most > 42 else most)
    _kv8.check((out[blind].double().cpu().numpy(), lse[blind].cpu().numpy()), [a[blind] for a in ref])
