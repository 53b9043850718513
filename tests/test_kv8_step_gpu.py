"""Places, append and attention together, as a serving loop runs them: eagerly, captured and replayed, on two streams, and beside the latent
cache's calls."""
import math

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B, workloads as W

pytestmark = pytest.mark.gpu
H, KV, D, BATCH, WIDTH = 8, 2, 128, 5, 12


class Loop:
    """The state of a serving loop; `step` runs the three calls on its buffers, in place."""

    def __init__(self, seed, places):
        g = np.random.default_rng(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.free = torch.from_numpy(g.permutation(BATCH * WIDTH + 5).astype(np.int32)).cuda()
        P = len(self.free)
        self.table, self.lens, self.new = torch.full((BATCH, WIDTH), -7, **i32), torch.zeros(BATCH, **i32), torch.zeros(BATCH, **i32)
        self.begin, self.places = torch.zeros(1, **i32), places
        self.pools = [torch.full((P, KV, 64, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scales = [torch.full((P, KV), float("nan"), device="cuda") for _ in range(2)]
        self.q, self.k, self.v = (torch.zeros((places, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, KV, KV))
        self.out, self.lse = torch.zeros((places, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((places, H), device="cuda")
        # the oracle's cache
        self.ref = _kv8.Cache(seed, [0] * BATCH, KV, D, width=WIDTH, spare=P)
        self.ref_values = [np.full((P, KV, 64, D), np.nan) for _ in range(2)]
        self.ref_scales = [np.full((P, KV), np.nan) for _ in range(2)]
        self.ref_begin = 0

    def step(self):
        slot_map, _, q_start, after, counts = B.splash_kv_slots(self.table, self.lens, self.new, self.free, self.begin, self.places)
        B.splash_kv8_append(self.k, self.v, slot_map, *self.pools, *self.scales)
        B.splash_kv8_attention(self.q, *self.pools, *self.scales, self.table, after, softmax_scale=1 / math.sqrt(D), q_start=q_start, max_q_rows=self.places,
                               out=self.out, lse=self.lse)
        self.lens.copy_(after)
        self.begin.copy_(counts[3:])

    def feed(self, seed, new):
        g = torch.Generator().manual_seed(seed)
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.x = [torch.randn(t.shape, generator=g).to(torch.bfloat16) for t in (self.q, self.k, self.v)]
        for t, x in zip((self.q, self.k, self.v), self.x):
            t.copy_(x)
        self.out.fill_(5.0), self.lse.fill_(5.0)

    def check(self, new):
        ref, rows = self.ref, sum(new)
        got = _kv8.slots(ref.table, ref.lens, new, self.free.cpu().numpy(), self.ref_begin, self.places)
        ref.table, ref.lens, self.ref_begin = got[0], got[4], int(got[5][3])
        assert np.array_equal(self.table.cpu().numpy(), ref.table) and np.array_equal(self.lens.cpu().numpy(), ref.lens) and int(self.begin) == self.ref_begin
        for k in range(2):
            self.ref_values[k], self.ref_scales[k] = _kv8.append(self.x[1 + k].double().numpy(), got[1], self.ref_values[k], self.ref_scales[k])
            assert np.array_equal(_kv8.E4M3[self.pools[k].cpu().numpy()], self.ref_values[k], equal_nan=True)
            ref.codes[k], ref.scales[k] = self.pools[k].cpu().numpy(), self.scales[k].cpu().numpy()
        expected = _kv8.attention(ref, self.x[0].double().numpy()[:rows], got[3], 1 / math.sqrt(D), out_eps=2.0 ** -8)
        _kv8.check((self.out[:rows].double().cpu().numpy(), self.lse[:rows].cpu().numpy()), expected)
        assert (self.out[rows:] == 5).all() and (self.lse[rows:] == 5).all()


STEPS = [[100, 3, 64, 1, 0], [1, 1, 1, 1, 1], [1, 1, 1, 0, 130], [70, 1, 2, 63, 1], [1, 1, 1, 1, 1], [8, 4, 1, 1, 3]]


def test_a_serving_loop():
    loop = Loop(1, 180)
    for k, new in enumerate(STEPS):
        loop.feed(k, new)
        loop.step()
        loop.check(new)


def test_captured_and_replayed():
    warm = Loop(2, 180)
    warm.feed(0, STEPS[0])
    warm.step()                                # the first call of each kind lies outside the capture
    loop, other = Loop(3, 180), Loop(4, 180)
    graphs = []
    for x in (loop, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.step()
        graphs.append(graph)
    for k, new in enumerate(STEPS):            # two graphs by turns, lengths and inputs changed in place
        for x, graph in ((loop, graphs[0]), (other, graphs[1])):
            x.feed(10 * k + (x is other), new)
            graph.replay()
        for x in (loop, other):
            x.check(new)


def test_two_streams_at_once():
    loops, streams = [Loop(5, 180), Loop(6, 180)], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k, new in enumerate(STEPS):
        for x in loops:
            x.feed(k, new)
        torch.cuda.synchronize()
        for x, s in zip(loops, streams):
            with torch.cuda.stream(s):
                x.step()
        torch.cuda.synchronize()
        for x in loops:
            x.check(new)


def test_a_given_stream():
    loop, s = Loop(7, 180), torch.cuda.Stream()
    loop.feed(0, STEPS[0])
    torch.cuda.synchronize()
    slot_map, _, q_start, after, counts = B.splash_kv_slots(loop.table, loop.lens, loop.new, loop.free, loop.begin, 180, stream=s)
    B.splash_kv8_append(loop.k, loop.v, slot_map, *loop.pools, *loop.scales, stream=s)
    B.splash_kv8_attention(loop.q, *loop.pools, *loop.scales, loop.table, after, softmax_scale=1 / math.sqrt(D), q_start=q_start, max_q_rows=180, out=loop.out, lse=loop.lse,
                           stream=s)
    s.synchronize()
    loop.lens.copy_(after), loop.begin.copy_(counts[3:])
    loop.check(STEPS[0])


def test_refused_requests_leave_the_cache_alone():
    loop = Loop(8, 180)
    loop.feed(0, [100, 3, 64, 1, 0])
    loop.begin.fill_(len(loop.free) - 2)       # two pages: enough for the first request alone
    slot_map, _, q_start, after, counts = B.splash_kv_slots(loop.table, loop.lens, loop.new, loop.free, loop.begin, 180)
    B.splash_kv8_append(loop.k, loop.v, slot_map, *loop.pools, *loop.scales)
    assert counts.tolist() == [168, 2, 3, len(loop.free)] and after.tolist() == [100, 0, 0, 0, 0]
    touched = sorted(loop.free[-2:].tolist())
    rest = [p for p in range(len(loop.free)) if p not in touched]
    assert (loop.pools[0][rest] == 0x7F).all() and loop.scales[0][rest].isnan().all() and not loop.scales[0][touched].isnan().any()


def test_places_for_the_latent_cache():
    # the same table and slot map place bf16 rows of the latent cache, which splash_mla_decode then reads
    g = np.random.default_rng(9)
    lens = [70, 1, 200]
    w = W.make_workload("places", 99, lens, H=16)
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table = torch.full((3, 6), -1, dtype=torch.int32, device="cuda")
    free = torch.from_numpy(g.permutation(20).astype(np.int32)).cuda()
    slot_map, positions, q_start, after, counts = B.splash_kv_slots(table, torch.zeros_like(new), new, free, torch.zeros(1, dtype=torch.int32, device="cuda"), sum(lens))
    assert positions.tolist() == [t for n in lens for t in range(n)] and counts.tolist() == [sum(lens), 7, 0, 7]
    dw = B.DeviceWorkload(w)
    rows = torch.cat([dw.kv_pool[dw.block_table[i, :(n + 63) // 64].long()].flatten(0, 1)[:n] for i, n in enumerate(lens)])
    pool = torch.full((20, 64, 576), float("nan"), dtype=torch.bfloat16, device="cuda")
    pool.view(-1, 576)[slot_map] = rows
    a = dw.decode()
    b = B.splash_mla_decode(dw.q, pool, table, after, softmax_scale=w.softmax_scale)
    assert (a[0] - b[0]).abs().max() <= 1e-2 and (a[1] - b[1]).abs().max() <= 1e-3


def test_scratch_belongs_to_the_given_stream():
    """Memory of the current stream's pool may still be in use by what that stream has before it, which the given stream does not wait for."""
    cache = _kv8.Cache([3], [700, 4000], 2, 128)
    tensors = cache.cuda()
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def allocated(stream):
        return sum(s["allocated_size"] + s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)

    here, there = allocated(torch.cuda.current_stream()), allocated(side)
    with torch.cuda.stream(torch.cuda.default_stream()):
        B.splash_kv8_attention(q, *tensors, softmax_scale=1.0, out=out, lse=lse, stream=side)
    assert allocated(side) > there and allocated(torch.cuda.current_stream()) == here
    B.splash_kv8_attention(q, *tensors, softmax_scale=1.0, out=out, lse=lse, stream=torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert torch.isfinite(lse).all()
