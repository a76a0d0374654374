"""tdk_rope, tdk_kv_create_rope, tdk_round_create_rope and tdk_kv_rotate: what the host refuses, with no device; the plain forms pinned."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

import kv_helpers as kh
import rope_helpers as rh
from paper_2604_03143_amd import tdk
from test_kv_args import batch, refused

P = 1 << 20      # an aligned address: nothing here is ever read


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(tdk.LIB_PATH):
        from paper_2604_03143_amd import _build
        _build.build(force=True)
    return tdk.load()


def rope(**kw):
    return tdk.rope(**{**dict(scaling=tdk.ROPE_SCALE_TURNS, factor=8.0, original_len=8192, low=1.0, high=4.0), **kw})


def make(fmt=tdk.KV_BF16, rp=None, **kw):
    return tdk.tdk_kv_create_rope(tdk.model(1, **kw), rp or rope(), fmt)


def io(**kw):
    return tdk.kv_rotate_io(**{**dict(k=P, k_stride=1024, k_out=2 * P, k_out_stride=1024, q=P, q_stride=5120, n_q_heads=40, q_out=2 * P, q_out_stride=5120), **kw})


BAD = [(dict(rotary_dim=0), tdk.ERR_UNSUPPORTED), (dict(rotary_dim=24), tdk.ERR_UNSUPPORTED), (dict(rotary_dim=144), tdk.ERR_UNSUPPORTED),
       (dict(rotary_dim=-16), tdk.ERR_UNSUPPORTED), (dict(scaling=4), tdk.ERR_UNSUPPORTED), (dict(scaling=-1), tdk.ERR_UNSUPPORTED),
       (dict(factor=0.99), tdk.ERR_INVALID_ARG), (dict(factor=math.inf), tdk.ERR_INVALID_ARG), (dict(factor=math.nan), tdk.ERR_INVALID_ARG),
       (dict(scaling=tdk.ROPE_SCALE_LINEAR, factor=0.5), tdk.ERR_INVALID_ARG), (dict(original_len=0), tdk.ERR_INVALID_ARG), (dict(original_len=math.inf), tdk.ERR_INVALID_ARG),
       (dict(low=0.0), tdk.ERR_INVALID_ARG), (dict(low=4.0), tdk.ERR_INVALID_ARG), (dict(high=math.inf), tdk.ERR_INVALID_ARG), (dict(high=math.nan), tdk.ERR_INVALID_ARG),
       (dict(magnitude=0.0), tdk.ERR_INVALID_ARG), (dict(magnitude=-1.0), tdk.ERR_INVALID_ARG), (dict(magnitude=math.nan), tdk.ERR_INVALID_ARG),
       (dict(magnitude=2e6), tdk.ERR_INVALID_ARG)]


@pytest.mark.parametrize("kw,status", BAD)
def test_create_refuses(kw, status):
    refused(lambda: make(rp=rope(**kw)), status, "rope")
    refused(lambda: tdk.tdk_round_create_rope(tdk.model(1), rope(**kw), [0], [0], [], [], []), status, "rope")


def test_more_that_create_refuses(lib):
    refused(lambda: make(rp=rope(scaling=tdk.ROPE_SCALE_INDEX), rope_theta=1.0), say="rope_theta")
    refused(lambda: make(head_dim=64), tdk.ERR_UNSUPPORTED)
    refused(lambda: make(fmt=2), tdk.ERR_UNSUPPORTED, "format")
    refused(lambda: tdk.tdk_round_create_rope(tdk.model(1), rope(rotary_dim=64), [0], [0], [], [], []), tdk.ERR_UNSUPPORTED, "whole heads")
    m, out = tdk.model(1), C.c_void_p(5)
    assert lib.tdk_kv_create_rope(C.byref(m), None, 0, C.byref(out)) == tdk.ERR_INVALID_ARG and not out
    out = C.c_void_p(5)
    assert lib.tdk_round_create_rope(C.byref(m), None, None, 0, None, 0, C.byref(out)) == tdk.ERR_INVALID_ARG and not out
    assert lib.tdk_kv_create_rope(C.byref(m), C.byref(rope()), 0, None) == tdk.ERR_INVALID_ARG
    assert lib.tdk_kv_create_rope(None, C.byref(rope()), 0, C.byref(out)) == tdk.ERR_INVALID_ARG


def test_fields_that_a_scaling_does_not_use_are_not_looked_at():
    nan = math.nan
    make(rp=tdk.rope(scaling=tdk.ROPE_SCALE_NONE, factor=nan, original_len=nan, low=nan, high=nan))
    make(rp=tdk.rope(scaling=tdk.ROPE_SCALE_LINEAR, factor=2.0, original_len=-1, low=nan, high=nan))


@pytest.mark.parametrize("kw", [dict(k=None), dict(k_out=None), dict(q=None), dict(q_out=None), dict(k=P + 8), dict(k_out=P + 2), dict(q=P + 4), dict(q_out=2 * P + 8),
                                dict(k_stride=1016), dict(k_out_stride=1028), dict(q_stride=5112), dict(q_out_stride=1 << 41), dict(k_stride=-1024),
                                dict(n_q_heads=0), dict(n_q_heads=-1), dict(n_q_heads=1 << 17), dict(k_out=P, k_out_stride=1032), dict(q_out=P, q_out_stride=5128)])
def test_rotation_refused(kw):
    refused(lambda: tdk.tdk_kv_rotate(make(), batch(), io(**kw)))


@pytest.mark.parametrize("kw,status", [(dict(n_seqs=-1), tdk.ERR_INVALID_ARG), (dict(n_tokens=-1), tdk.ERR_INVALID_ARG), (dict(q_start=None), tdk.ERR_INVALID_ARG),
                                       (dict(seq_len=None), tdk.ERR_INVALID_ARG), (dict(q_start=P + 2), tdk.ERR_INVALID_ARG), (dict(seq_len=P + 1), tdk.ERR_INVALID_ARG),
                                       (dict(n_tokens=(1 << 30) + 1), tdk.ERR_UNSUPPORTED), (dict(n_seqs=(1 << 30) + 1), tdk.ERR_UNSUPPORTED),
                                       (dict(n_tokens=1 << 24), tdk.ERR_UNSUPPORTED)])
def test_batches_refused(kw, status):
    refused(lambda: tdk.tdk_kv_rotate(make(), batch(**kw), io()), status)


def test_null_arguments(lib):
    kv = make()
    for i in range(3):
        args = [kv.handle, C.byref(batch()), C.byref(io())]
        args[i] = None
        assert lib.tdk_kv_rotate(*args, None) == tdk.ERR_INVALID_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_right_arguments_get_as_far_as_the_device():
    kv = make()
    none = dict(k=None, k_out=None)
    for a, b in ((io(), batch()), (io(**none), batch()), (io(q=None, q_out=None), batch()), (io(), batch(block_table=None, table_stride=0, max_len=0)),
                 (io(), batch(n_seqs=0, q_start=None)), (io(q=None, q_out=None, **none), batch(q_start=None)), (io(k_out=P, q_out=P), batch())):
        refused(lambda: tdk.tdk_kv_rotate(kv, b, a), say="device")


def test_page_bytes_of_eight_bits():
    assert tdk.tdk_kv_page_bytes(make(tdk.KV_MXFP8)) == 16 * 8 * 132
    assert tdk.tdk_kv_page_bytes(tdk.tdk_kv_create(tdk.model(1, num_kv_heads=3, page_tokens=32), tdk.KV_MXFP8)) == 32 * 3 * 132


# ---- the plain forms that the GPU tests compare with, pinned where they can be ----

def test_frequencies_by_hand():
    f = rh.frequencies(1e4, 128)
    assert f[0] == 1.0 and math.isclose(f[63], 1e4 ** (-126 / 128))
    assert np.allclose(rh.frequencies(1e4, 64, "linear", 4.0), 1e4 ** (-np.arange(32) / 32) / 4, rtol=1e-15)
    g = rh.frequencies(5e5, 128, "turns", 8.0, 8192, 1.0, 4.0)
    f = rh.frequencies(5e5, 128)
    turns = 8192 * f / (2 * math.pi)
    assert (g[turns > 4] == f[turns > 4]).all() and np.allclose(g[turns < 1], f[turns < 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and ((g[mid] < f[mid]) & (g[mid] > f[mid] / 8)).all()
    g = rh.frequencies(1e4, 128, "index", 32.0, 4096, 1.0, 32.0)      # pairs 20 to 46: 64 ln(4096 / (32 * 2 pi)) / ln 1e4 = 20.9, 64 ln(4096 / 2 pi) / ln 1e4 = 45.03
    f = rh.frequencies(1e4, 128)
    assert (g[:21] == f[:21]).all() and g[21] < f[21] and np.allclose(g[46:], f[46:] / 32, rtol=1e-15) and g[45] > f[45] / 32
    assert math.isclose(g[33], f[33] / 32 * 0.5 + f[33] * 0.5)


def test_rotation_of_part_of_the_head():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3, 2, 128)).astype(np.float32)
    assert np.array_equal(rh.rotate(x, [0, 7, 12345], rh.frequencies(1e6), 128, False), kh.rotate(x, [0, 7, 12345], 1e6, False))
    assert np.array_equal(rh.rotate(x, [0, 7, 12345], rh.frequencies(1e6), 128, True), kh.rotate(x, [0, 7, 12345], 1e6, True))
    f = rh.frequencies(1e6, 64)
    y = rh.rotate(x, [0, 7, 12345], f, 64, False)
    assert np.array_equal(y[..., 64:], x[..., 64:])
    z = (x[..., :32] + 1j * x[..., 32:64]).astype(np.complex128) * np.exp(1j * np.outer([0, 7, 12345], f))[:, None, :]
    assert np.allclose(y[..., :32], z.real, atol=1e-6) and np.allclose(y[..., 32:64], z.imag, atol=1e-6)
    again = rh.rotate(rh.rotate(x, [3, 4, 5], f, 64, True, 1.5), [3, 4, 5], f, 64, True, 1.5, back=True)
    assert np.allclose(again, x, atol=1e-5)


def test_eight_bit_grid_by_hand():
    x = torch.zeros(1, 128, dtype=torch.float64)
    x[0, :8] = torch.tensor([448.0, 464.0, 17.0, 19.0, -0.001, 2.0 ** -10, 3 * 2.0 ** -10, -240.0])
    x[0, 32:34] = torch.tensor([464.5, 1.0])                      # above 1.8125 * 2^8: the next power of two, 232.25 between 224 and 240
    x[0, 64] = float("nan")
    code, byte = rh.to8(x)
    assert byte[0].tolist() == [127, 128, 255, 3]
    assert rh.from8(code, byte)[0, :8].tolist() == [448, 448, 16, 20, -2.0 ** -9, 0, 2.0 ** -8, -240]
    assert rh.from8(code, byte)[0, 32:34].tolist() == [480, 1.0]
    assert torch.isnan(rh.from8(code, byte)[0, 64:96]).all() and (rh.from8(code, byte)[0, 96:] == 0).all()
    v = torch.randn(4, 128).abs() + 0.1
    c, b = rh.to8(v)
    assert ((rh.from8(c, b) / v - 1).abs() <= 2.0 ** -4).all()
    assert torch.equal(rh.GRID8[:127], torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
