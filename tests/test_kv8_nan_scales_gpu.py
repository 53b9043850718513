"""A key scale that is NaN: the rows that see a token of the page have NaN, in out and lse; every other row's are as they were."""
import math

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [[4, 3], [1, 5], [150, 70], [140, 1]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_that_do_not_see_the_page_keep_their_sums(rows, D, bad):
    lens, heads, group = [194, 130], 2, 2                    # the last pages, of two tokens each, begin at 192 and 128
    cache = _kv8.Cache([51, D], lens, heads, D)
    T = sum(rows)
    q = torch.from_numpy(np.random.default_rng(51).normal(size=(T, heads * group, D))).to(torch.bfloat16)
    q_start = [0, rows[0], T]
    kw = dict(softmax_scale=1 / math.sqrt(D), q_start=torch.tensor(q_start, dtype=torch.int32, device="cuda"), max_q_rows=max(rows))
    ref = [a.copy() for a in _kv8.attention(cache, q.double().numpy(), q_start, 1 / math.sqrt(D), out_eps=2.0 ** -8)]
    sees = np.zeros((T, heads * group), bool)
    for i, n in enumerate(lens):
        first = (n - 1) // 64 * 64
        cache.scales[0][cache.table[i, first // 64], 1] = bad                  # of the second key head
        for k in range(rows[i]):
            sees[q_start[i] + k, group:] = n - rows[i] + k >= first
    out, lse = (x.double().cpu().numpy() for x in B.splash_kv8_attention(q.cuda(), *cache.cuda(), **kw))
    ro, rl, to, tl = ref
    assert sees.any() and (~sees).any()
    assert np.isfinite(lse[~sees]).all() and (np.abs(lse - rl) <= tl)[~sees].all(), "a sum of a row that does not see the page"
    assert np.isfinite(out[~sees]).all() and (np.abs(out - ro) <= to)[~sees].all()
    assert not np.isfinite(lse[sees]).any() and np.isnan(out[sees]).all()
