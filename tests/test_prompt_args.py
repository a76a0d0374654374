"""tdk_prompt_attend: what the host refuses, with no device, and what it computes itself."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import prompt_helpers as ph
from paper_2604_03143_amd import tdk
from test_kv_args import make, refused

P = 1 << 20      # an aligned address: nothing here is ever read


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(tdk.LIB_PATH):
        from paper_2604_03143_amd import _build
        _build.build(force=True)
    return tdk.load()


def batch(**kw):
    return tdk.prompt_batch(**{**dict(n_seqs=3, n_q=5, n_k=50, max_len=100, q_start=P, k_start=P), **kw})


def io(**kw):
    return tdk.prompt_attend_io(**{**dict(q=P, q_stride=5120, n_q_heads=40, k=P, k_stride=1024, v=P, v_stride=1024, scale=0.1, out=P, out_stride=5120, lse=P, workspace=P,
                                          workspace_bytes=1 << 40), **kw})


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(q=P + 8), dict(out=P + 8), dict(k=P + 2), dict(v=P + 8), dict(q_stride=5112),
                                dict(out_stride=5124), dict(k_stride=1016), dict(v_stride=1028), dict(k_stride=(1 << 24) + 8), dict(v_stride=1 << 30), dict(n_q_heads=0),
                                dict(n_q_heads=36), dict(n_q_heads=-8), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(window=-1), dict(n_sink=-1),
                                dict(part_out=P), dict(part_lse=P), dict(part_out=P + 4, part_lse=P), dict(part_out=P, part_lse=P + 2), dict(lse=P + 2), dict(workspace=None),
                                dict(workspace=P + 128), dict(workspace_bytes=0)])
def test_refused(kw):
    kv = make()
    assert tdk.tdk_prompt_attend_workspace_bytes(kv, batch(max_len=100000), 40) > 0
    refused(lambda: tdk.tdk_prompt_attend(kv, batch(max_len=100000), io(**kw)))


@pytest.mark.parametrize("kw,status", [(dict(n_seqs=-1), tdk.ERR_INVALID_ARG), (dict(n_q=-1), tdk.ERR_INVALID_ARG), (dict(n_k=-1), tdk.ERR_INVALID_ARG),
                                       (dict(max_len=-1), tdk.ERR_INVALID_ARG), (dict(q_start=None), tdk.ERR_INVALID_ARG), (dict(k_start=None), tdk.ERR_INVALID_ARG),
                                       (dict(q_start=P + 2), tdk.ERR_INVALID_ARG), (dict(k_start=P + 1), tdk.ERR_INVALID_ARG), (dict(n_q=(1 << 30) + 1), tdk.ERR_UNSUPPORTED),
                                       (dict(n_k=(1 << 30) + 1), tdk.ERR_UNSUPPORTED), (dict(n_seqs=(1 << 30) + 1), tdk.ERR_UNSUPPORTED),
                                       (dict(n_q=1 << 27), tdk.ERR_UNSUPPORTED), (dict(n_seqs=1 << 21, n_q=1 << 21), tdk.ERR_UNSUPPORTED)])
def test_batches_refused(kw, status):
    refused(lambda: tdk.tdk_prompt_attend(make(), batch(**kw), io()), status)


def test_null_arguments(lib):
    kv = make()
    for i in range(3):
        args = [kv.handle, C.byref(batch()), C.byref(io())]
        args[i] = None
        assert lib.tdk_prompt_attend(*args, None) == tdk.ERR_INVALID_ARG
    assert lib.tdk_prompt_attend_workspace_bytes(None, C.byref(batch()), 40) == 0
    assert lib.tdk_prompt_attend_workspace_bytes(kv.handle, None, 40) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_right_arguments_get_as_far_as_the_device():
    kv = make()
    for b, a in ((batch(), io()), (batch(n_seqs=0, q_start=None, k_start=None), io(q=None, out=None)), (batch(n_q=0), io()), (batch(n_k=0), io(k=None, v=None)),
                 (batch(), io(lse=None, out_f32=True)), (batch(), io(part_out=P, part_lse=P, window=5, n_sink=3))):
        refused(lambda: tdk.tdk_prompt_attend(kv, b, a), say="device")


def test_workspace_depends_on_sizes_alone():
    kv = make()
    need = lambda **kw: tdk.tdk_prompt_attend_workspace_bytes(kv, batch(q_start=None, k_start=None, **kw), 40)   # noqa: E731
    assert need(n_seqs=0) == need(n_q=0) == 0
    assert need(n_seqs=25, n_q=25000, n_k=25000, max_len=1000) == 0            # enough rows for the whole device
    assert need(n_seqs=1, n_q=1, n_k=100000, max_len=100000) > 0
    assert tdk.tdk_prompt_attend_workspace_bytes(kv, batch(), 36) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_the_workspace_serves_every_window():
    """A window makes a call shorter, and cuts it otherwise: never into more parts than the workspace that was asked for has room for."""
    rng = np.random.default_rng(11)
    for _ in range(4000):
        heads, seqs = int(rng.choice([1, 2, 3, 8])), int(2 ** rng.uniform(0, 9))
        group, length = int(rng.choice([1, 4, 5, 8, 16])), int(2 ** rng.uniform(0, 18))
        tokens = int(rng.choice([seqs, seqs * 3, seqs + 7, seqs * 40, seqs * 300]))
        kv, qd = make(num_kv_heads=heads), heads * group * 128
        b = batch(n_seqs=seqs, n_q=tokens, n_k=seqs * length if seqs * length < 1 << 30 else 1 << 20, max_len=length)
        need = tdk.tdk_prompt_attend_workspace_bytes(kv, b, heads * group)
        a = io(n_q_heads=heads * group, q_stride=qd, out_stride=qd, window=int(2 ** rng.uniform(0, 18)), n_sink=int(rng.integers(0, 9)), workspace_bytes=need)
        refused(lambda: tdk.tdk_prompt_attend(kv, b, a), say="device")


def test_plain_form_against_softmax():
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, h, 128, generator=g, dtype=torch.float64) for n, h in ((5, 4), (9, 2), (9, 2)))
    out, lse, _, _ = ph.attend([(2, 6), (3, 3)], q, k, v, 0.1)
    s = q[1, 3] @ k[:6, 1].T * 0.1
    assert torch.allclose(out[1, 3], torch.softmax(s, -1) @ v[:6, 1]) and torch.allclose(lse[1, 3], torch.logsumexp(s, -1))
    assert torch.allclose(out[2, 0], v[6, 0])
    out, lse, _, _ = ph.attend([(5, 3)], q, k, v, 0.1, window=1, sink=1)
    assert (out[:2] == 0).all() and (lse[:2] == -torch.inf).all() and torch.allclose(out[3, 2], torch.softmax(q[3, 2] @ k[:2, 1].T * 0.1, -1) @ v[:2, 1])
    v[1] = float("inf")
    out, _, _, _ = ph.attend([(3, 3)], q, k, v, 0.1)
    assert torch.isfinite(out[0]).all() and (out[1:3] == float("inf")).all()


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
def test_the_workspace_of_eight_bit_pages_serves_every_window():
    from test_kv_args import batch as kv_batch, cache, io as kv_io
    rng = np.random.default_rng(12)
    for _ in range(4000):
        heads, seqs = int(rng.choice([1, 2, 3, 8])), int(2 ** rng.uniform(0, 11))
        group, length = int(rng.choice([1, 4, 5, 8, 16])), int(2 ** rng.uniform(0, 18))
        tokens = int(rng.choice([seqs, seqs * 3, seqs + 7, seqs * 40]))
        kv, qd = make(tdk.KV_MXFP8, num_kv_heads=heads), heads * group * 128
        b = kv_batch(n_seqs=seqs, n_tokens=tokens, max_len=length)
        need = tdk.tdk_kv_attend_workspace_bytes(kv, b, heads * group)
        a = kv_io(n_q_heads=heads * group, q_stride=qd, out_stride=qd, window=int(2 ** rng.uniform(0, 18)), n_sink=int(rng.integers(0, 9)), workspace_bytes=need)
        refused(lambda: tdk.tdk_kv_attend(kv, cache(), b, a), say="device")
