"""Outputs of decode, sparse decode, merge and the DOP layout changes on a given stream: what the caller does not bring lies in that stream's
memory (the current stream's pool hands out blocks that the current stream may still have work for)."""
import numpy as np
import pytest

from paper_2609_37626_b200 import workloads as W

pytestmark = pytest.mark.gpu


def pool_of(tensor):
    import torch
    at = tensor.untyped_storage().data_ptr()
    return next(s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"])


def calls():
    import torch
    from paper_2609_37626_b200 import binding
    w = W.make_workload("streams", 4100, [70, 200, 5], H=16)
    dw = binding.DeviceWorkload(w)
    yield "decode", lambda **kw: binding.splash_mla_decode(dw.q, dw.kv_pool, dw.block_table, dw.seq_lens, softmax_scale=w.softmax_scale, **kw)
    sw = W.make_workload("streams", 4101, [70, 200, 5], H=16, kv_dtype=2)
    sel, cnt = (torch.from_numpy(a).cuda() for a in W.select_tokens(4101, sw.seq_lens, 40))
    ds = binding.DeviceWorkload(sw)
    yield "sparse", lambda **kw: binding.splash_mla_decode_sparse(ds.q, ds.kv_pool, ds.block_table, ds.seq_lens, sel, cnt, softmax_scale=sw.softmax_scale, **kw)
    g = np.random.default_rng(4)
    parts, lses = torch.from_numpy(g.normal(size=(3, 40, 64)).astype(np.float32)).cuda(), torch.from_numpy(g.normal(size=(3, 40)).astype(np.float32)).cuda()
    yield "merge", lambda **kw: binding.splash_lse_merge(parts, lses, **kw)
    x, row = torch.from_numpy(g.normal(size=(9, 4, 64)).astype(np.float32)).cuda(), torch.tensor([3, 0, 8], dtype=torch.int32, device="cuda")
    yield "pack", lambda **kw: (binding.splash_dop_pack_rows(x, None, row, **kw),)
    yield "swap", lambda **kw: (binding.splash_dop_swap_outer(x, **kw),)


@pytest.mark.parametrize("which", ["decode", "sparse", "merge", "pack", "swap"])
def test_outputs_lie_in_the_memory_of_the_calls_stream(which):
    import torch
    side = torch.cuda.Stream()
    call = dict(calls())[which]
    here = call()
    torch.cuda.synchronize()
    there = call(stream=side)
    torch.cuda.synchronize()
    assert {pool_of(t) for t in here} == {torch.cuda.current_stream().cuda_stream}
    assert {pool_of(t) for t in there} == {side.cuda_stream}
    assert all(torch.equal(a, b) for a, b in zip(here, there))
