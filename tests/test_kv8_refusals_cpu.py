"""What the operators around the 8-bit cache refuse, on the host, before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import _kv8
from paper_2609_37626_b200 import binding as B, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


P = 0x10000


def cache(**kw):
    c = B.Kv8Cache(struct_size=ctypes.sizeof(B.Kv8Cache), num_pages=8, num_kv_heads=2, head_dim=128, page_size=64, k_pool=P, v_pool=P, k_scales=P, v_scales=P,
                   k_page_stride=2 * 8192, k_head_stride=8192, v_page_stride=2 * 8192, v_head_stride=8192, k_scale_stride=2, v_scale_stride=2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def query(**kw):
    s = B.Kv8Query(struct_size=ctypes.sizeof(B.Kv8Query), num_requests=3, num_rows=3, num_heads=8, max_q_rows=1, dtype=0, out_dtype=0, q_row_stride=1024,
                   q_head_stride=128, out_row_stride=1024, out_head_stride=128, lse_row_stride=8, block_table_stride=4, table_width=4, softmax_scale=0.1)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_struct_sizes():
    assert ctypes.sizeof(B.Kv8Cache) == 104 and ctypes.sizeof(B.Kv8Query) == 88


def attend(lib, c, s, q=P, ws=P, ws_bytes=1 << 40, q_start=None, table=P):
    vp = ctypes.c_void_p
    return lib.splash_kv8_attention(ctypes.byref(c), ctypes.byref(s), vp(q), vp(table), vp(P), q_start, None, None, vp(P), vp(P), vp(ws), ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(struct_size=4), dict(num_pages=0), dict(k_pool=None), dict(v_scales=None), dict(k_pool=P + 8), dict(k_scales=P + 2),
                                 dict(k_page_stride=8200), dict(v_head_stride=64), dict(v_head_stride=8200), dict(k_scale_stride=1)])
def test_bad_caches(lib, bad):
    assert attend(lib, cache(**bad), query()) == B.SPLASH_INVALID_ARG
    vp = ctypes.c_void_p
    assert lib.splash_kv8_append(ctypes.byref(cache(**bad)), 0, 4, vp(P), 256, 128, vp(P), 256, 128, vp(P), None) == B.SPLASH_INVALID_ARG
    assert lib.splash_kv8_attention_workspace_bytes(ctypes.byref(cache(**bad)), ctypes.byref(query())) == 0


@pytest.mark.parametrize("other", [dict(head_dim=96), dict(head_dim=256), dict(page_size=16), dict(num_kv_heads=0)])
def test_unsupported_caches(lib, other):
    assert attend(lib, cache(**other), query()) == B.SPLASH_UNSUPPORTED
    assert lib.splash_last_error()


@pytest.mark.parametrize("bad", [dict(struct_size=80), dict(num_requests=-1), dict(num_rows=-1), dict(num_heads=7), dict(num_heads=0), dict(max_q_rows=0), dict(q_row_stride=1028),
                                 dict(q_head_stride=64), dict(out_head_stride=100), dict(out_row_stride=8), dict(lse_row_stride=7), dict(block_table_stride=3),
                                 dict(softmax_scale=float("nan")), dict(table_width=-1), dict(num_rows=4)])
def test_bad_queries(lib, bad):
    assert attend(lib, cache(), query(**bad)) == B.SPLASH_INVALID_ARG
    assert lib.splash_last_launch_count() == 0


@pytest.mark.parametrize("other", [dict(dtype=2), dict(dtype=7), dict(out_dtype=1), dict(num_rows=1 << 31), dict(num_heads=4096)])
def test_unsupported_queries(lib, other):
    assert attend(lib, cache(), query(**other), q_start=ctypes.c_void_p(P)) == B.SPLASH_UNSUPPORTED


def test_bad_pointers_and_empty_work(lib):
    assert attend(lib, cache(), query(), q=0) == B.SPLASH_INVALID_ARG
    assert attend(lib, cache(), query(), q=P + 2) == B.SPLASH_INVALID_ARG
    assert attend(lib, cache(), query(), ws=P + 128) == B.SPLASH_INVALID_ARG
    assert attend(lib, cache(), query(), table=0) == B.SPLASH_INVALID_ARG
    assert attend(lib, cache(), query(num_requests=0, num_rows=0), q=0) == B.SPLASH_OK
    assert attend(lib, cache(), query(num_rows=0), q=0, q_start=ctypes.c_void_p(P)) == B.SPLASH_OK
    assert lib.splash_last_launch_count() == 0


def test_append_refusals(lib):
    vp = ctypes.c_void_p

    def call(dtype=0, n=4, k=P, kr=256, kh=128, vr=256, vh=128, slots=P):
        return lib.splash_kv8_append(ctypes.byref(cache()), dtype, n, vp(k), kr, kh, vp(P), vr, vh, vp(slots), None)
    assert call(dtype=2) == B.SPLASH_UNSUPPORTED
    for bad in (dict(n=-1), dict(k=0), dict(k=P + 8), dict(kr=257), dict(kh=64), dict(vr=64), dict(vh=132), dict(slots=0), dict(slots=P + 4)):
        assert call(**bad) == B.SPLASH_INVALID_ARG, bad
    assert call(n=0, k=0) == B.SPLASH_OK and lib.splash_last_launch_count() == 0


def test_slots_refusals(lib):
    vp = ctypes.c_void_p
    good = dict(n=2, lens=P, new=P + 0x100, free=P + 0x200, num_free=4, begin=P + 0x300, table=P + 0x400, stride=4, width=4, places=8, slots=P + 0x500,
                positions=P + 0x600, q_start=P + 0x700, after=P + 0x800, counts=P + 0x900)

    def call(**kw):
        a = dict(good, **kw)
        return lib.splash_kv_slots(a["n"], vp(a["lens"]), vp(a["new"]), vp(a["free"]), a["num_free"], vp(a["begin"]), vp(a["table"]), a["stride"], a["width"],
                                   a["places"], vp(a["slots"]), vp(a["positions"]), vp(a["q_start"]), vp(a["after"]), vp(a["counts"]), None)
    for bad in (dict(n=-1), dict(num_free=-1), dict(width=-1), dict(places=-1), dict(stride=3), dict(lens=0), dict(counts=0), dict(slots=0), dict(begin=0),
                dict(slots=P + 0x504), dict(lens=P + 2),
                dict(after=P), dict(q_start=P + 0x104), dict(counts=P + 0x300), dict(positions=P + 0x520), dict(table=P + 0x200)):
        assert call(**bad) == B.SPLASH_INVALID_ARG, bad
    assert call(n=16385) == B.SPLASH_UNSUPPORTED
    assert call(num_free=1 << 31) == B.SPLASH_UNSUPPORTED
    assert lib.splash_last_launch_count() == 0


def test_the_binding_wants_gpu_tensors_that_fit():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)      # noqa: E731
    pools = [torch.zeros((4, 2, 64, 128), dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros((4, 2)) for _ in range(2)]
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(AssertionError, match="GPU"):
        B.splash_kv8_attention(q, *pools, *scales, i32(3, 2), i32(3), softmax_scale=1.0)
    with pytest.raises(AssertionError, match="GPU"):
        B.splash_kv8_append(q[:, :2], q[:, :2], torch.zeros(3, dtype=torch.int64), *pools, *scales)
    with pytest.raises(AssertionError, match="GPU"):
        B.splash_kv_slots(i32(3, 2), i32(3), i32(3), i32(4), i32(1), 4)
    with pytest.raises(TypeError):
        B.splash_kv8_attention(q, *pools, *scales, i32(3, 2), i32(3))
    for bad in (dict(pools=[pools[0], pools[1][:3]]), dict(pools=[pools[0].float(), pools[1]]), dict(pools=[pools[0][:, :, :32], pools[1][:, :, :32]]),
                dict(pools=[pools[0].transpose(2, 3), pools[1].transpose(2, 3)]), dict(scales=[scales[0].double(), scales[1]]), dict(scales=[scales[0][:, :1], scales[1]]),
                dict(table=i32(2, 2)), dict(table=i32(3, 2).long()), dict(lens=i32(3).long()), dict(q=q[:, :, :64]), dict(q_start=i32(3)), dict(max_q_rows=0)):
        a = dict(q=q, pools=pools, scales=scales, table=i32(3, 2), lens=i32(3))
        a.update({k: v for k, v in bad.items() if k in a})
        with pytest.raises(AssertionError):
            B.splash_kv8_attention(a["q"], *a["pools"], *a["scales"], a["table"], a["lens"], softmax_scale=1.0,
                                   **{k: v for k, v in bad.items() if k not in a})
    with pytest.raises(AssertionError):
        B.splash_kv8_append(q[:, :2], q[:2, :2], torch.zeros(3, dtype=torch.int64), *pools, *scales)
    with pytest.raises(AssertionError):
        B.splash_kv8_append(q[:, :2], q[:, :2], i32(3), *pools, *scales)


def test_the_plain_forms():
    # the table of codes against torch's, the grid against the table, scales against their definition
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, _kv8.E4M3, equal_nan=True)
    x = np.random.default_rng(0).normal(size=4000) * np.exp2(np.random.default_rng(1).integers(-14, 10, 4000))
    x = np.concatenate([x, [0.0, 448.0, 460.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, -17.0]])
    assert np.array_equal(_kv8.to_grid(x), torch.from_numpy(np.clip(x, -448, 448)).to(torch.float32).to(torch.float8_e4m3fn).double().numpy())
    for most in (448.0, 448.1, 1.0, 0.875, 0.8750001, 1e-40, 0.0, 3e38):
        s = _kv8.power_of_two_scale(most)
        assert most <= 448 * s and (s == 2.0 ** -100 or most > 448 * s / 2)
