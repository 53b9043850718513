"""Block tables and slot maps against a loop over the requests: whole numbers, equal."""
import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu


def make(seed, batch, high, new_high, width_slack=2, spare=5, negative=False):
    g = np.random.default_rng(seed)
    lens, new = g.integers(0, high + 1, batch), g.integers(0, new_high + 1, batch)
    if negative:
        lens[::5], new[::7] = -3, -1
    width = max([-(-(max(int(a), 0) + max(int(b), 0)) // 64) for a, b in zip(lens, new)] + [1]) + width_slack
    table = g.integers(0, 1000, (batch, width)).astype(np.int32)
    free = (1000 + g.permutation(sum(-(-int(max(a, 0) + max(b, 0)) // 64) for a, b in zip(lens, new)) + spare + 4)).astype(np.int32)
    return table, lens.astype(np.int32), new.astype(np.int32), free


def run(table, lens, new, free, begin, places, **kw):
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()       # noqa: E731
    t = cu(table)
    got = B.splash_kv_slots(t, cu(lens), cu(new), cu(free), torch.tensor([begin], dtype=torch.int32, device="cuda"), places, **kw)
    torch.cuda.synchronize()
    return [t.cpu().numpy()] + [x.cpu().numpy() for x in got]


def same(got, ref):
    for name, x, y in zip(("block_table", "slot_map", "positions", "q_start", "new_seq_lens", "counts"), got, ref):
        assert x.dtype == y.dtype and np.array_equal(x, y), name


@pytest.mark.parametrize("batch,high,new_high", [(1, 0, 1), (1, 63, 1), (1, 64, 200), (3, 130, 70), (33, 300, 1), (64, 8192, 1), (511, 2000, 40), (700, 100, 130), (5, 100, 9000)])
@pytest.mark.parametrize("seed", [0, 1])
def test_all_served(batch, high, new_high, seed):
    table, lens, new, free = make(seed, batch, high, new_high)
    places = int(new.sum()) + 37 * seed
    ref = _kv8.slots(table, lens, new, free, 4, places)
    assert ref[-1][2] == 0
    same(run(table, lens, new, free, 4, places), ref)


@pytest.mark.parametrize("case", ["pages", "width", "places", "negative", "no free list", "begin behind it", "begin negative", "nothing new"])
def test_refusals_and_odd_inputs(case):
    table, lens, new, free = make(11, 90, 500, 150, negative=case == "negative")
    begin, places = 4, int(np.maximum(new, 0).sum()) + 10
    if case == "pages":
        free = free[:60]
    elif case == "width":
        table = np.ascontiguousarray(table[:, :6])
    elif case == "places":
        places = places // 2
    elif case == "no free list":
        free = free[:0]
        begin = 0
    elif case == "begin behind it":
        begin = len(free) + 5
    elif case == "begin negative":
        begin = -2
    elif case == "nothing new":
        new[:] = 0
    ref = _kv8.slots(table, lens, new, free, begin, places)
    assert (ref[-1][2] > 0) == (case not in ("negative", "nothing new"))
    same(run(table, lens, new, free, begin, places), ref)


def test_no_requests_and_no_places():
    empty = np.zeros(0, np.int32)
    got = run(np.zeros((0, 4), np.int32), empty, empty, np.arange(5, dtype=np.int32), 2, 9)
    assert (got[1] == -1).all() and (got[2] == -1).all() and got[3].tolist() == [0] and got[5].tolist() == [0, 0, 0, 2]
    table, lens, new, free = make(3, 4, 100, 0)
    same(run(table, lens, new, free, 0, 0), _kv8.slots(table, lens, new, free, 0, 0))


def test_sums_behind_the_range_of_places():
    # lengths that add up to more than 2^31: nobody behind that is served, the sums stop at 2^31 - 1
    lens, new = np.array([5, 0, 7, 1], np.int32), np.array([3, 2 ** 31 - 1, 2 ** 31 - 1, 1], np.int32)
    table, free = np.full((4, 3), 9, np.int32), np.arange(50, dtype=np.int32)
    ref = _kv8.slots(table, lens, new, free, 0, 8)
    assert ref[5].tolist() == [2 ** 31 - 1, 0, 3, 0]
    same(run(table, lens, new, free, 0, 8), ref)


def test_the_most_requests():
    n = 16384
    g = np.random.default_rng(5)
    lens, new = g.integers(0, 200, n).astype(np.int32), g.integers(0, 4, n).astype(np.int32)
    table = g.integers(0, 1000, (n, 4)).astype(np.int32)
    free = np.arange(n, dtype=np.int32)
    same(run(table, lens, new, free, 7, int(new.sum()) + 3), _kv8.slots(table, lens, new, free, 7, int(new.sum()) + 3))


def test_a_view_of_a_wider_table_and_given_outputs():
    table, lens, new, free = make(21, 40, 400, 90)
    wide = np.full((40, table.shape[1] + 5), -5, np.int32)
    wide[:, 2:2 + table.shape[1]] = table
    places = int(new.sum()) + 1
    ref = _kv8.slots(table, lens, new, free, 0, places)
    cu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()       # noqa: E731
    t = cu(wide)
    outs = [torch.empty(places, dtype=torch.int64, device="cuda")] + [torch.empty(n, dtype=torch.int32, device="cuda") for n in (places, 41, 40, 4)]
    got = B.splash_kv_slots(t[:, 2:2 + table.shape[1]], cu(lens), cu(new), cu(free), cu(np.zeros(1, np.int32)), places, slot_map=outs[0], positions=outs[1],
                            q_start=outs[2], new_seq_lens=outs[3], counts=outs[4])
    assert all(a is b for a, b in zip(got, outs))
    after = t.cpu().numpy()
    assert (after[:, :2] == -5).all() and (after[:, 2 + table.shape[1]:] == -5).all()
    same([after[:, 2:2 + table.shape[1]]] + [x.cpu().numpy() for x in got], ref)
    with pytest.raises(B.SplashError, match="overlaps"):
        B.splash_kv_slots(t[:, 2:2 + table.shape[1]], outs[3], cu(new), cu(free), cu(np.zeros(1, np.int32)), places, new_seq_lens=outs[3])
