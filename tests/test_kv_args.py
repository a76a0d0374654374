"""tdk_kv_*: what the host refuses, before anything is asked of a device (so all of it can be had without one), and what it computes itself."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk

P = 1 << 20      # an aligned address: nothing here is ever read


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(tdk.LIB_PATH):
        from paper_2604_03143_amd import _build
        _build.build(force=True)
    return tdk.load()


def make(fmt=tdk.KV_BF16, **kw):
    return tdk.tdk_kv_create(tdk.model(1, **kw), fmt)


def cache(**kw):
    return tdk.kv_cache(**{**dict(k=P, v=P, pool_pages=7), **kw})


def batch(**kw):
    return tdk.kv_batch(**{**dict(n_seqs=3, n_tokens=5, max_len=100, q_start=P, seq_len=P, block_table=P, table_stride=9), **kw})


def rows(**kw):
    return tdk.kv_rows(**{**dict(k=P, v=P, k_stride=1024, v_stride=1024), **kw})


def io(**kw):
    return tdk.kv_attend_io(**{**dict(q=P, q_stride=5120, n_q_heads=40, scale=0.1, out=P, out_stride=5120, lse=P, workspace=P, workspace_bytes=1 << 40), **kw})


def refused(f, status=tdk.ERR_INVALID_ARG, say=None):
    with pytest.raises(tdk.TdkError) as e:
        f()
    assert e.value.status == status and e.value.detail
    assert say is None or say in e.value.detail


@pytest.mark.parametrize("kw,status", [(dict(head_dim=64), tdk.ERR_UNSUPPORTED), (dict(page_tokens=8), tdk.ERR_UNSUPPORTED),
                                       (dict(num_kv_heads=9), tdk.ERR_UNSUPPORTED), (dict(rope_theta=-1.0), tdk.ERR_INVALID_ARG),
                                       (dict(rope_style=2), tdk.ERR_INVALID_ARG), (dict(fmt=2), tdk.ERR_UNSUPPORTED)])
def test_create_refuses(kw, status):
    refused(lambda: make(**kw), status)


def test_null_arguments(lib):
    kv = make()
    assert lib.tdk_kv_create(None, 0, C.byref(C.c_void_p())) == tdk.ERR_INVALID_ARG
    assert lib.tdk_kv_create(C.byref(tdk.model(1)), 0, None) == tdk.ERR_INVALID_ARG
    lib.tdk_kv_destroy(None)
    assert lib.tdk_kv_page_bytes(None) == 0 and lib.tdk_kv_attend_workspace_bytes(None, C.byref(batch()), 40) == 0
    assert lib.tdk_kv_attend_workspace_bytes(kv.handle, None, 40) == 0
    for f, last in ((lib.tdk_kv_append, rows()), (lib.tdk_kv_read, rows()), (lib.tdk_kv_attend, io())):
        args = [kv.handle, C.byref(cache()), C.byref(batch()), C.byref(last)]
        for i in range(4):
            assert f(*[None if j == i else a for j, a in enumerate(args)], None) == tdk.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(n_tokens=-1), dict(max_len=-1), dict(table_stride=-1), dict(q_start=None), dict(seq_len=None),
                                dict(block_table=None), dict(q_start=P + 2), dict(seq_len=P + 1), dict(block_table=P + 2)])
def test_batches_refused_by_every_call(kw):
    kv = make()
    refused(lambda: tdk.tdk_kv_append(kv, cache(), batch(**kw), rows()))
    refused(lambda: tdk.tdk_kv_read(kv, cache(), batch(**kw), rows()))
    refused(lambda: tdk.tdk_kv_attend(kv, cache(), batch(**kw), io()))


@pytest.mark.parametrize("kw", [dict(pool_pages=-1), dict(pool_pages=1 << 31), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 4)])
def test_caches_refused_by_every_call(kw):
    kv = make(tdk.KV_MXFP4)
    refused(lambda: tdk.tdk_kv_append(kv, cache(**kw), batch(), rows()))
    refused(lambda: tdk.tdk_kv_read(kv, cache(**kw), batch(), rows()))
    refused(lambda: tdk.tdk_kv_attend(kv, cache(**kw), batch(), io()))


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(k_stride=1016), dict(v_stride=1028), dict(k_stride=-1024),
                                dict(k_stride=1 << 41), dict(q=P), dict(q_out=P), dict(q=P, q_out=2 * P, q_stride=5120, q_out_stride=5120),
                                dict(q=P, q_out=2 * P, q_stride=5112, q_out_stride=5120, n_q_heads=40),
                                dict(q=P, q_out=2 * P, q_stride=5120, q_out_stride=5124, n_q_heads=40),
                                dict(q=P, q_out=P, q_stride=5120, q_out_stride=5128, n_q_heads=40),
                                dict(q=P + 4, q_out=2 * P, q_stride=5120, q_out_stride=5120, n_q_heads=40)])
def test_rows_refused(kw):
    refused(lambda: tdk.tdk_kv_append(make(), cache(), batch(), rows(**kw)))


def test_read_takes_no_queries():
    refused(lambda: tdk.tdk_kv_read(make(), cache(), batch(), rows(q=P, q_out=2 * P, q_stride=5120, q_out_stride=5120, n_q_heads=40)), say="queries")


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 8), dict(q_stride=5112), dict(out_stride=5124), dict(n_q_heads=0),
                                dict(n_q_heads=36), dict(n_q_heads=-8), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(n_sink=-1),
                                dict(part_out=P), dict(part_lse=P), dict(part_out=P + 4, part_lse=P), dict(part_out=P, part_lse=P + 2), dict(hole=P + 2),
                                dict(lse=P + 2), dict(workspace=None), dict(workspace=P + 128), dict(workspace_bytes=0)])
def test_attention_refused(kw):
    kv = make()
    assert tdk.tdk_kv_attend_workspace_bytes(kv, batch(max_len=100000), 40) > 0
    refused(lambda: tdk.tdk_kv_attend(kv, cache(), batch(max_len=100000), io(**kw)))


def test_too_many_tokens():
    kv = make()
    for b in (batch(n_tokens=(1 << 30) + 1), batch(table_stride=1 << 27)):
        refused(lambda: tdk.tdk_kv_append(kv, cache(), b, rows()), tdk.ERR_UNSUPPORTED)
        refused(lambda: tdk.tdk_kv_attend(kv, cache(), b, io()), tdk.ERR_UNSUPPORTED)
    refused(lambda: tdk.tdk_kv_attend(kv, cache(), batch(n_tokens=1 << 26), io()), tdk.ERR_UNSUPPORTED, "grid")
    # a launch has fewer than 2^32 threads: 256 per token moved, 256 per block of query rows and KV head (here 2^21 sequences of one block, 8 heads)
    for f in (tdk.tdk_kv_append, tdk.tdk_kv_read):
        refused(lambda: f(kv, cache(), batch(n_tokens=1 << 24), rows(q=None, q_out=None)), tdk.ERR_UNSUPPORTED, "launch")
    refused(lambda: tdk.tdk_kv_attend(kv, cache(), batch(n_seqs=1 << 21, n_tokens=1 << 21), io()), tdk.ERR_UNSUPPORTED, "grid")


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_right_arguments_get_as_far_as_the_device():
    kv = make()
    for f in (lambda: tdk.tdk_kv_append(kv, cache(), batch(), rows()), lambda: tdk.tdk_kv_read(kv, cache(), batch(), rows()),
              lambda: tdk.tdk_kv_attend(kv, cache(), batch(), io()), lambda: tdk.tdk_kv_append(kv, cache(), batch(n_seqs=0), rows()),
              lambda: tdk.tdk_kv_attend(kv, cache(pool_pages=0, k=None, v=None), batch(n_tokens=0, q_start=None), io(q=None, out=None))):
        refused(f, say="device")


def test_page_bytes():
    assert tdk.tdk_kv_page_bytes(make()) == 16 * 8 * 256
    assert tdk.tdk_kv_page_bytes(make(tdk.KV_MXFP4, num_kv_heads=3, page_tokens=32)) == 32 * 3 * 68


def test_workspace_depends_on_sizes_alone():
    kv = make()
    need = lambda **kw: tdk.tdk_kv_attend_workspace_bytes(kv, batch(q_start=None, seq_len=None, block_table=None, **kw), 40)   # noqa: E731
    assert need(n_seqs=0) == need(n_tokens=0) == 0
    assert need(n_seqs=250, n_tokens=250, max_len=100) == 0                     # enough sequences for the whole device
    assert need(n_seqs=1, n_tokens=1, max_len=100000) > 0
    assert tdk.tdk_kv_attend_workspace_bytes(kv, batch(), 36) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4])
def test_the_workspace_serves_every_window(fmt):
    """A window makes a call shorter, and cuts it otherwise: never into more parts than the workspace that was asked for has room for."""
    rng = np.random.default_rng(11)
    for _ in range(3000):
        heads, seqs = int(rng.choice([1, 2, 3, 8])), int(2 ** rng.uniform(0, 11))
        group, length = int(rng.choice([1, 4, 5, 8, 16])), int(2 ** rng.uniform(0, 18))
        tokens = int(rng.choice([seqs, seqs * 3, seqs + 7, seqs * 40]))
        kv = make(fmt, num_kv_heads=heads)
        b = batch(n_seqs=seqs, n_tokens=tokens, max_len=length)
        qd = heads * group * 128
        need = tdk.tdk_kv_attend_workspace_bytes(kv, b, heads * group)
        a = io(n_q_heads=heads * group, q_stride=qd, out_stride=qd, window=int(2 ** rng.uniform(0, 18)), n_sink=int(rng.integers(0, 9)), workspace_bytes=need)
        refused(lambda: tdk.tdk_kv_attend(kv, cache(), b, a), say="device")


# ---- the plain forms that the GPU tests compare with, pinned where they can be ----

def test_four_bit_grid_by_hand():
    x = torch.zeros(1, 128, dtype=torch.float64)
    x[0, :12] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0, 0.26, -0.2, 5.1, 6.9])
    x[0, 32:35] = torch.tensor([7.0, -7.0, 1.0])                  # from 1.75 * 2^2 on the next power of two
    x[0, 64] = float("inf")
    code, byte = kh.to4(x)
    assert byte[0].tolist() == [127, 128, 255, 1]
    assert kh.from4(code, byte)[0, :12].tolist() == [4, 0, 1, 1, 2, 2, 4, -4, .5, 0, 6, 6]
    assert kh.from4(code, byte)[0, 32:35].tolist() == [8, -8, 1]
    assert torch.isnan(kh.from4(code, byte)[0, 64:96]).all() and (kh.from4(code, byte)[0, 96:] == 0).all()
    T = 16
    pages = kh.pack4(code.reshape(1, 1, 1, 128).expand(2, T, 3, 128), byte.reshape(1, 1, 1, 4).expand(2, T, 3, 4), T)
    assert pages.shape == (2, 3, T * 68)
    c2, b2 = kh.unpack4(pages, T)
    assert torch.equal(c2, code.reshape(1, 1, 1, 128).expand(2, T, 3, 128)) and torch.equal(b2, byte.reshape(1, 1, 1, 4).expand(2, T, 3, 4))


def test_plain_attention_against_softmax():
    b = kh.Batch([(3, 2), (0, 1)], 16, 1)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(b.pool_pages, 16, 2, 128, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(b.n, 4, 128, generator=g, dtype=torch.float64)
    out, lse, _, _ = kh.attend(b, k, v, q, 0.1)
    p = int(b.table[0, 0])
    s = q[1, 3] @ k[p, :5, 1].T * 0.1
    assert torch.allclose(out[1, 3], torch.softmax(s, -1) @ v[p, :5, 1]) and torch.allclose(lse[1, 3], torch.logsumexp(s, -1))
    out, lse, _, _ = kh.attend(b, k, v, q, 0.1, hole=[(0, 4), (0, 9)])
    assert torch.allclose(out[1, 3], v[p, 4, 1]) and (out[2] == 0).all() and (lse[2] == -torch.inf).all() and (out[0] == 0).all()


def test_rotation_against_complex_numbers():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3, 2, 128)).astype(np.float32)
    got = kh.rotate(x, [0, 7, 12345], 1e6, False)
    assert np.array_equal(got[0], x[0])
    z = (x[..., :64] + 1j * x[..., 64:]).astype(np.complex128) * np.exp(1j * np.outer([0, 7, 12345], 1e6 ** (-np.arange(64) / 64)))[:, None, :]
    assert np.allclose(got[..., :64], z.real, atol=1e-6) and np.allclose(got[..., 64:], z.imag, atol=1e-6)
