"""tdk_kv_attend and tdk_kv_read with 4-bit blocks of every exponent: beyond bf16's range a value is infinite."""
import math

import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk
from test_gpu_kv import bf, bits, handle, stream

pytestmark = pytest.mark.gpu


def bf16_of(code, byte):
    """What a 4-bit row is in bf16: beyond its range infinity."""
    return kh.from4(code, byte).float().to(torch.bfloat16)


def run(b, fmt, H, group, dk, dv, q, scale, window=0, sink=0, hole=None, part=(None, None), max_len=None):
    kv, Hq = handle(fmt, H, b.T), H * group
    out, lse = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:2], 9.0, device="cuda")
    batch = b.struct(tdk, max_len)
    need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, Hq)
    space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    hd = None if hole is None else torch.tensor(hole, dtype=torch.int32, device="cuda")
    keep = [dk.cuda(), dv.cuda(), q.cuda(), *(None if p is None else p.cuda() for p in part)]
    io = tdk.kv_attend_io(keep[2], Hq * 128, Hq, scale, out, Hq * 128, lse, space, need, window, sink, hd, *keep[3:])
    tdk.tdk_kv_attend(kv, tdk.kv_cache(keep[0], keep[1], b.pool_pages), batch, io, stream())
    torch.cuda.synchronize()
    return out.cpu().double(), lse.cpu().double()


def close(got, want, tol):
    same = (got == want) | (torch.isnan(got) & torch.isnan(want)) | ((got - want).abs() <= torch.nan_to_num(tol, nan=0.0, posinf=0.0))
    assert same.all(), (int((~same).sum()), got.numel(), got[~same][:4], want[~same][:4])


@pytest.mark.parametrize("byte", [253, 254, 255])
@pytest.mark.parametrize("lengths,group", [([(30, 3)], 3), ([(30, 4), (5, 1)], 5), ([(30, 40)], 3), ([(3, 150)], 2), ([(600, 30)], 4)])
def test_blocks_beyond_bf16_reach_the_rows_that_see_them_only(byte, lengths, group):
    """4 * 2^126 and 2 * 2^127 are infinite in bf16.  The token that holds such a block of V is seen by some rows and not by others."""
    H, T = 2, 16
    b, g = kh.Batch(lengths, T, 3), torch.Generator().manual_seed(4)
    codes = [kh.to4(torch.randn(b.pool_pages, T, H, 128, generator=g)) for _ in range(2)]
    h, n = lengths[0]
    at = b.slot(0, h + max(1, n // 2))
    codes[1][0][at][:, 32:64] = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15] * 2, dtype=torch.uint8)
    codes[1][1][at][:, 1] = byte
    dk, dv = (kh.pack4(*x, T) for x in codes)
    q = bf(torch.randn(b.n, H * group, 128, generator=g))
    scale = 1 / math.sqrt(128)
    k, v = (bf16_of(*x).double() for x in codes)
    want, wlse, mass, big = kh.attend(b, k, v, q.double(), scale)
    got, glse = run(b, tdk.KV_MXFP4, H, group, dk, dv, q, scale)
    tol, ltol = kh.tolerance(want, wlse, mass, big, 700)
    before = max(1, n // 2)
    assert torch.isfinite(want[:before]).all() and not torch.isfinite(want[before]).all()
    close(got, want, tol)
    close(glse, wlse, ltol)


@pytest.mark.parametrize("n_new", [4, 60])
def test_the_largest_values_that_are_appended(n_new):
    """V of about 3e38, finite in bf16: its block's nearest 4-bit value is 2^128, which rows before the token do not meet."""
    H, group, T = 2, 4, 16
    b, g = kh.Batch([(20, n_new)], T, 3), torch.Generator().manual_seed(4)
    k, v = (bf(torch.randn(b.n, H * 128, generator=g)) for _ in range(2))
    v[n_new // 2] = 3.0e38
    kv = handle(tdk.KV_MXFP4, H, T)
    pk, pv = (torch.zeros(b.pool_pages, H, T * 68, dtype=torch.uint8, device="cuda") for _ in range(2))
    kd, vd = k.cuda(), v.cuda()
    tdk.tdk_kv_append(kv, tdk.kv_cache(pk, pv, b.pool_pages), b.struct(tdk), tdk.kv_rows(kd, vd, H * 128, H * 128), stream())
    torch.cuda.synchronize()
    q = bf(torch.randn(b.n, H * group, 128, generator=g))
    planes = [bf16_of(*kh.unpack4(x.cpu(), T)).double() for x in (pk, pv)]
    want, wlse, mass, big = kh.attend(b, *planes, q.double(), 0.1)
    got, glse = run(b, tdk.KV_MXFP4, H, group, pk, pv, q, 0.1)
    tol, ltol = kh.tolerance(want, wlse, mass, big, 100)
    assert torch.isfinite(got[:n_new // 2]).all()
    close(got, want, tol)
    close(glse, wlse, ltol)


@pytest.mark.parametrize("T", [16, 32])
def test_every_block_exponent_is_read_back(T):
    """All 256 bytes with all sixteen codes, bit for bit: from half of 2^-127, a bf16 number without a leading one, to infinity and NaN."""
    H, n = 2, 32
    b = kh.Batch([(0, n)], T, 3)
    code = torch.arange(16, dtype=torch.uint8).repeat(8).expand(b.pool_pages, T, H, 128).contiguous()
    byte = torch.zeros(b.pool_pages, T, H, 4, dtype=torch.uint8)
    for t in range(n):
        byte[b.slot(0, t)] = torch.arange(8 * t, 8 * t + 8, dtype=torch.uint8).reshape(H, 4)
    pk = kh.pack4(code, byte, T).cuda()
    pv = kh.pack4(code ^ 8, byte, T).cuda()
    kv = handle(tdk.KV_MXFP4, H, T)
    out = [torch.zeros(n, H * 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tdk.tdk_kv_read(kv, tdk.kv_cache(pk, pv, b.pool_pages), b.struct(tdk), tdk.kv_rows(*out, H * 128, H * 128), stream())
    torch.cuda.synchronize()
    for got, c in zip(out, (code, code ^ 8)):
        full = bf16_of(c, byte)
        want = torch.stack([full[b.slot(0, t)] for t in range(n)]).reshape(n, -1)
        got, nan = got.cpu(), torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan)
        assert torch.equal(bits(got)[~nan], bits(want)[~nan])
