"""tdk_kv_attend with values near the end of bf16's range: the sums behind a result stay finite where the result is."""
import math

import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk
from test_gpu_kv import FORMATS, bf, handle, stream

pytestmark = pytest.mark.gpu
T, H, GROUP = 16, 2, 4


def attend(fmt, b, k, v, q, scale, part=(None, None)):
    """On the device and in 64 bits: out, lse, and the second's tolerance (kh.tolerance)."""
    if fmt == tdk.KV_MXFP4:
        dk, dv = (kh.pack4(*kh.to4(x.float()), T) for x in (k, v))
        k, v = (kh.from4(*kh.unpack4(x, T)) for x in (dk, dv))
    else:
        dk, dv = k, v
    want, wlse, mass, big = kh.attend(b, k.double(), v.double(), q.double(), scale, 0, 0, None, *(None if p is None else p.double() for p in part))
    kv, Hq = handle(fmt, H, T), H * GROUP
    out, lse = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:2], 9.0, device="cuda")
    batch = b.struct(tdk)
    need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, Hq)
    space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    keep = [dk.cuda(), dv.cuda(), q.cuda(), *(None if p is None else p.cuda() for p in part)]
    io = tdk.kv_attend_io(keep[2], Hq * 128, Hq, scale, out, Hq * 128, lse, space, need, 0, 0, None, *keep[3:])
    tdk.tdk_kv_attend(kv, tdk.kv_cache(keep[0], keep[1], b.pool_pages), batch, io, stream())
    torch.cuda.synchronize()
    tol, ltol = kh.tolerance(want, wlse, mass, big, max(h + n for h, n in b.lengths))
    assert torch.isfinite(want).all()
    assert ((out.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wlse).abs() <= ltol).all()


@FORMATS
@pytest.mark.parametrize("lengths,far", [([(250, 1)], 130), ([(250, 3), (9, 1)], 140), ([(200, 40)], 130), ([(3000, 1)], 2900), ([(700, 50)], 400)])
@pytest.mark.parametrize("value", [1.0e37, 2.5e38])
def test_a_large_value_whose_score_comes_late(fmt, lengths, far, value):
    """One token of the first sequence has the score 4 (all scores are exact), the others have zero; its V is large.  The reference point is
    still that of the tokens before it, and its weight e^4: times the value more than fp32 holds, while the result, its share of the
    value, is finite."""
    b, g = kh.Batch(lengths, T, 3), torch.Generator().manual_seed(4)
    k = torch.zeros(b.pool_pages, T, H, 128)
    v = torch.randn(b.pool_pages, T, H, 128, generator=g)
    k[b.slot(0, far)] = 0.5
    v[b.slot(0, far)][:, 64:96] = value
    q = torch.ones(b.n, H * GROUP, 128)
    attend(fmt, b, bf(k), bf(v), bf(q), 1 / 16)


@FORMATS
def test_two_large_parts_joined(fmt):
    """Both parts hold 3e38 (in 4 bits the nearest value below): their shares are added, not the two themselves."""
    b, g = kh.Batch([(40, 1), (3, 2)], T, 3), torch.Generator().manual_seed(4)
    k = torch.randn(b.pool_pages, T, H, 128, generator=g)
    v = torch.full((b.pool_pages, T, H, 128), 3.0e38 if fmt == tdk.KV_BF16 else 2.5e38)
    q = torch.randn(b.n, H * GROUP, 128, generator=g)
    part = torch.full((b.n, H * GROUP, 128), 3.0e38), torch.full((b.n, H * GROUP), math.log(20.0))
    attend(fmt, b, bf(k), bf(v), bf(q), 1 / math.sqrt(128), part)
