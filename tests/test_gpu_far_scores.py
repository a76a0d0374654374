"""Attention whose scores lie far from zero, and scales that leave one key all the weight, in the step kernels of prompts and of pages: bounds of far_helpers, which zeros
and exchanged rows do not pass (test_far_bounds.py)."""
import pytest
import torch

import far_helpers as fh
import kv_helpers as kh
import prompt_helpers as ph
import rope_helpers as rh
from paper_2604_03143_amd import tdk
from test_gpu_kv import stream
from test_gpu_kv8 import check_attend
from test_gpu_kv_values import run

pytestmark = pytest.mark.gpu
H = 2


def run_prompt(lengths, q, k, v, scale, window=0, sink=0, part=(None, None)):
    Hq, n, m = q.shape[1], q.shape[0], k.shape[0]
    d = [x.flatten(1).cuda() for x in (q, k, v)]
    part = [None if p is None else p.cuda() for p in part]
    starts = [torch.tensor([0, *torch.tensor(x).cumsum(0).tolist()], dtype=torch.int32, device="cuda") for x in zip(*lengths)]
    kv, batch = tdk.tdk_kv_create(tdk.model(1, k.shape[1])), tdk.prompt_batch(len(lengths), n, m, max(x for _, x in lengths), *starts)
    need = tdk.tdk_prompt_attend_workspace_bytes(kv, batch, Hq)
    space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.full((n, Hq * 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, Hq), 9.0, device="cuda")
    wide = [x.shape[1] for x in d]
    tdk.tdk_prompt_attend(kv, batch, tdk.prompt_attend_io(d[0], wide[0], Hq, d[1], wide[1], d[2], wide[2], scale, out, wide[0], lse, space, need, window, sink, *part), stream())
    torch.cuda.synchronize()
    return out.cpu().double().reshape(n, Hq, 128), lse.cpu().double(), need


def parts(n, Hq, lse):
    """A part over other tokens, of about the weight of the rows' own; some have none."""
    g = torch.Generator().manual_seed(6)
    po, pl = torch.randn(n, Hq, 128, generator=g), (lse + torch.randn(n, Hq, generator=g)).float()
    pl[::3, ::2] = -torch.inf
    return po, pl


WIDE = [(300, 300)] * 17


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lengths,group", [([(200, 200)], 5), ([(40, 900), (3, 77), (130, 130)], 5), (WIDE, 8), ([(5, 5000)], 5), ([(70, 3000)], 4)],
                         ids=["one", "chunks", "wide", "parts", "rows-in-parts"])
@pytest.mark.parametrize("window,sink,join", [(0, 0, False), (60, 3, False), (0, 0, True), (100, 5, True)])
def test_prompts_far_from_zero(sign, lengths, group, window, sink, join):
    n, m = (sum(x) for x in zip(*lengths))
    q, k, v = fh.rows(n, H * group, m, H, 11, sign)
    args = (lengths, q.double().cuda(), k.double().cuda(), v.double().cuda(), fh.SCALE, window, sink)
    part = (None, None)
    if join:
        part = parts(n, H * group, ph.attend(*args)[1].cpu())
    want, wlse, mass, big = ph.attend(*args, *(None if p is None else p.double().cuda() for p in part))
    got, glse, _ = run_prompt(lengths, q, k, v, fh.SCALE, window, sink, part)
    tol, ltol = (t.cpu() for t in kh.tolerance(want, wlse, mass, big, max(x for _, x in lengths)))
    assert fh.wrong_shifted(got, want.cpu(), tol) == 0
    assert ((glse - wlse.cpu()).abs() <= ltol).all()


@pytest.mark.parametrize("scale", [2.0 ** 12, 2.0 ** 20, -2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("lengths", [[(120, 120), (30, 300)], [(40, 3000)], [(1, 2000)]], ids=["short", "parts", "one-row"])
def test_prompts_with_one_key_to_a_row(scale, lengths):
    n, m = (sum(x) for x in zip(*lengths))
    q, k, v = fh.rows(n, H * 5, m, H, 12)
    sees, at = [], 0
    for a, b in lengths:
        sees += [range(at, at + b - a + t + 1) for t in range(a)]
        at += b
    bounds = fh.steep_all(q.double(), k.double(), v.double(), scale, sees)
    assert bounds[0].double().mean() > 0.9
    got, _, _ = run_prompt(lengths, q, k, v, scale)
    assert fh.wrong_steep(got, bounds) == 0


FORMATS = pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4, tdk.KV_MXFP8], ids=["bf16", "mxfp4", "mxfp8"])


def pages(fmt, b, k, v):
    """Rows of the sequences' tokens, one sequence behind the other, in pages of a format; and the values that those stand for, by page."""
    pk, pv = (torch.zeros(b.pool_pages, b.T, H, 128, dtype=torch.bfloat16) for _ in range(2))
    at = 0
    for s, (h, n) in enumerate(b.lengths):
        for j in range(h + n):
            pk[b.slot(s, j)], pv[b.slot(s, j)] = k[at], v[at]
            at += 1
    if fmt == tdk.KV_BF16:
        return pk, pv, pk.double(), pv.double()
    to, pack, back, split = (kh.to4, kh.pack4, kh.from4, kh.unpack4) if fmt == tdk.KV_MXFP4 else (rh.to8, rh.pack8, rh.from8, rh.unpack8)
    dk, dv = (pack(*to(x.float()), b.T) for x in (pk, pv))
    return dk, dv, *(back(*split(x, b.T)) for x in (dk, dv))


# rows of a sequence and KV head: many (the step kernels), up to 32, up to 16; and long ones, cut into parts
PAGED = pytest.mark.parametrize("lengths,group", [([(20, 70), (600, 40)], 4), ([(300, 5), (40, 5)], 5), ([(90, 1), (333, 1)], 5), ([(3000, 12)], 4), ([(3000, 1)], 5)],
                                ids=["many", "some", "few", "many-in-parts", "few-in-parts"])


@FORMATS
@PAGED
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("kw", [dict(), dict(window=60, sink=3), dict(window=50, sink=4, hole=True, join=True)], ids=["all", "window", "window-hole-join"])
def test_pages_far_from_zero(fmt, lengths, group, sign, kw):
    b = kh.Batch(lengths, 16, 2)
    q, k, v = fh.rows(b.n, H * group, sum(h + n for h, n in lengths), H, 13, sign)
    dk, dv, k64, v64 = pages(fmt, b, k, v)
    window, sink = kw.get("window", 0), kw.get("sink", 0)
    hole = [(max(0, h - 20), max(0, h - 20) + 11) for h, _ in lengths] if kw.get("hole") else None
    args, part = (b, k64, v64, q.double(), fh.SCALE, window, sink, hole), (None, None)
    if kw.get("join"):
        part = parts(b.n, H * group, kh.attend(*args)[1])
    want, wlse, mass, big = kh.attend(*args, *(None if p is None else p.double() for p in part))
    got, glse = run(b, fmt, H, group, dk, dv, q, fh.SCALE, window, sink, hole, part)
    tol, ltol = kh.tolerance(want, wlse, mass, big, max(h + n for h, n in lengths))
    assert fh.wrong_shifted(got, want, tol) == 0
    assert ((glse - wlse).abs() <= ltol).all()


@FORMATS
@PAGED
@pytest.mark.parametrize("scale", [2.0 ** 20, -2.0 ** 40])
def test_pages_with_one_key_to_a_row(fmt, lengths, group, scale):
    b = kh.Batch(lengths, 16, 3)
    q, k, v = fh.rows(b.n, H * group, sum(h + n for h, n in lengths), H, 14)
    dk, dv, k64, v64 = pages(fmt, b, k, v)
    flat = [torch.cat([torch.stack([x[b.slot(s, j)] for j in range(h + n)]) for s, (h, n) in enumerate(lengths)]) for x in (k64, v64)]
    first = [0]
    for h, n in lengths:
        first.append(first[-1] + h + n)
    bounds = fh.steep_all(q.double(), *flat, scale, [range(first[s], first[s] + p + 1) for s, p in b.positions()])
    assert bounds[0].double().mean() > 0.9
    got, _ = run(b, fmt, H, group, dk, dv, q, scale)
    assert fh.wrong_steep(got, bounds) == 0


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.1, 1.0, 3e-39])
@pytest.mark.parametrize("kw", [dict(), dict(window=30, sink=2, hole=[(3, 9), (5, 20)], join=True)], ids=["all", "window-hole-join"])
def test_scales_of_eight_bit_pages_with_many_rows(scale, kw):
    check_attend(2, 4, 16, [(50, 20), (20, 30)], scale=scale, **kw)
