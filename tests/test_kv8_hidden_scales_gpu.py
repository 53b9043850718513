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


# rows of one request each, and its context: the last page (or two) is hidden from the first rows.  Whole contexts and such as are cut and joined, one
# tile of rows and several
CHUNKS = [([150], [200], 4), ([300, 70], [300, 75], 1), ([90], [9000], 2)]


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
