"""Outputs that a call on a given stream allocates: they belong to that stream's memory.  Memory of the current stream's pool may still be
in use by what that stream has before it, which the given stream does not wait for."""
import math

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B

pytestmark = pytest.mark.gpu


def stream_of_memory(tensor):
    """The stream whose pool the tensor's memory lies in."""
    at = tensor.untyped_storage().data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def places(stream, lens=(70, 3), new=(1, 100), **kw):
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(5, 15, dtype=torch.int32, device="cuda")
    args = (table, ints(*lens), ints(*new), free, ints(0), 101 + 50_000)
    torch.cuda.synchronize()
    return B.splash_kv_slots(*args, stream=stream, **kw)


def attend(cache, q, stream, **kw):
    tensors = cache.cuda()
    torch.cuda.synchronize()
    return B.splash_kv8_attention(q, *tensors, softmax_scale=1 / math.sqrt(cache.D), stream=stream, **kw)


@pytest.mark.parametrize("given", [True, False])
def test_outputs_lie_in_the_memory_of_the_calls_stream(given):
    side = torch.cuda.Stream()
    cache = _kv8.Cache(1, [700, 90], 2, 128)
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    stream = side if given else None
    expected = side.cuda_stream if given else torch.cuda.current_stream().cuda_stream
    outs = (*places(stream), *attend(cache, q, stream))
    torch.cuda.synchronize()
    assert [stream_of_memory(t) for t in outs] == [expected] * 7


def test_outputs_that_are_given_stay_where_they_are():
    side = torch.cuda.Stream()
    cache = _kv8.Cache(2, [70, 90], 2, 64)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, counts = torch.empty_like(q), torch.empty(4, dtype=torch.int32, device="cuda")
    got, lse = attend(cache, q, side, out=out)
    more = places(side, counts=counts)
    torch.cuda.synchronize()
    assert got is out and more[4] is counts
    assert [stream_of_memory(t) for t in (lse, *more[:4])] == [side.cuda_stream] * 5


def test_the_current_stream_is_busy_with_freed_blocks():
    """Blocks as large as the outputs, freed while the current stream has still to write them: the call on the other stream is done long before."""
    side = torch.cuda.Stream()
    g = np.random.default_rng(3)
    cache = _kv8.Cache(3, [130, 64, 300], 4, 128)
    rows = [130, 64, 300]
    q = torch.from_numpy(g.normal(size=(sum(rows), 32, 128))).to(torch.bfloat16)
    q_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    kw = dict(q_start=torch.from_numpy(q_start).cuda(), max_q_rows=max(rows))
    qc = q.cuda()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.empty(qc.numel() * 2 + 4096, dtype=torch.uint8, device="cuda"), torch.empty(sum(rows) * 32 * 4, dtype=torch.uint8, device="cuda"),
              torch.empty(12 * 50_300, dtype=torch.uint8, device="cuda")]
    tensors = cache.cuda()
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    args = (table, ints(70, 3), ints(1, 100), torch.arange(5, 15, dtype=torch.int32, device="cuda"), ints(0), 101 + 50_000)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                  # about a tenth of a second
    for b in blocks:
        b.fill_(0x55)
    del b, blocks
    out, lse = B.splash_kv8_attention(qc, *tensors, softmax_scale=0.1, stream=side, **kw)
    slots = B.splash_kv_slots(*args, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    _kv8.check((out.double().cpu().numpy(), lse.cpu().numpy()), _kv8.attention(cache, q.double().numpy(), q_start, 0.1, out_eps=2.0 ** -8))
    ref = _kv8.slots(np.full((2, 4), -1, np.int32), [70, 3], [1, 100], np.arange(5, 15), 0, 101 + 50_000)
    for got, want in zip(slots, ref[1:]):
        assert np.array_equal(got.cpu().numpy(), want)
