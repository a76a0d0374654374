"""tdk_kv_append / tdk_kv_read / tdk_kv_attend on the GPU against plain forms in 64 bits: rows and 4-bit values bit for bit, attention by
tolerances that follow from its arithmetic (kv_helpers.tolerance)."""
import math

import numpy as np
import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def bf(x):
    return torch.as_tensor(x).to(torch.bfloat16)


def bits(t):
    return t.contiguous().view(torch.int16).cpu()


def handle(fmt, H, T, interleaved=False, theta=1.0e6):
    return tdk.tdk_kv_create(tdk.model(1, H, 128, T, theta, tdk.ROPE_INTERLEAVED if interleaved else tdk.ROPE_HALF), fmt)


def pools(fmt, pages, H, T, fill):
    if fmt == tdk.KV_BF16:
        return [torch.full((pages, T, H, 128), fill, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    return [torch.full((pages, H, T * 68), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]


# lengths: (earlier tokens, new tokens) per sequence
RAGGED = [(0, 1), (37, 0), (15, 18), (16, 16), (100, 3), (1, 1)]


def check_append(fmt, H, Hq, T, interleaved, theta, lengths, seed=1, fused=False, pad=0, spoil=None, values=None):
    g = torch.Generator().manual_seed(seed)
    b = kh.Batch(lengths, T, seed, pad_tokens=pad)
    if spoil:
        spoil(b)
    N, wide = b.n_tokens, (Hq + 2 * H) * 128
    x = bf(torch.randn(N, wide, generator=g))
    if values is not None:
        values(x[:, Hq * 128:])
    xd = x.cuda()
    parts = torch.split(xd, [Hq * 128, H * 128, H * 128], 1)
    if not fused:
        parts = [p.contiguous() for p in parts]
    q, k, v = parts
    kv, (pk, pv) = handle(fmt, H, T, interleaved, theta), pools(fmt, b.pool_pages, H, T, 7.0)
    before = [p.clone() for p in (pk, pv)]
    q_out = torch.full((N, Hq * 128 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    batch, cache = b.struct(tdk), tdk.kv_cache(pk, pv, b.pool_pages)
    rows = tdk.kv_rows(k, v, k.stride(0) if H else 0, v.stride(0), q=q, q_stride=q.stride(0), n_q_heads=Hq, q_out=q_out, q_out_stride=q_out.stride(0))
    tdk.tdk_kv_append(kv, cache, batch, rows, stream())
    torch.cuda.synchronize()
    # the expected cache
    xf = x.float().numpy()
    where = b.positions()
    pos = [p for _, p in where]
    n = len(where)
    want_q = bf(kh.rotate(xf[:n, :Hq * 128].reshape(n, Hq, 128), pos, theta, interleaved)) if n else None
    kr = kh.rotate(xf[:n, Hq * 128:(Hq + H) * 128].reshape(n, H, 128), pos, theta, interleaved) if n else None
    vr = x[:n, (Hq + H) * 128:].reshape(n, H, 128)
    seen = [i for i, (s, p) in enumerate(where) if p >= 0]
    for r in range(n):
        if r in seen:
            assert torch.equal(bits(q_out[r, :Hq * 128]), bits(want_q[r].reshape(-1)))
        else:
            assert (q_out[r] == 3.0).all()
    assert (q_out[n:] == 3.0).all() and (q_out[:, Hq * 128:] == 3.0).all()
    for plane, (got, old, new) in enumerate(zip((pk, pv), before, (kr, vr))):
        want = old.cpu().clone()
        if fmt == tdk.KV_MXFP4:
            codes, bytes_ = kh.unpack4(want, T)
            codes, bytes_ = codes.clone(), bytes_.clone()
            if n:
                c, e = kh.to4(torch.as_tensor(np.asarray(new) if plane == 0 else new.float().numpy()))
        for r in seen:
            slot = b.slot(*where[r])
            if slot is None:
                continue
            if fmt == tdk.KV_BF16:
                want[slot] = bf(kr[r]) if plane == 0 else vr[r]
            else:
                codes[slot], bytes_[slot] = c[r], e[r]
        if fmt == tdk.KV_MXFP4:
            want = kh.pack4(codes, bytes_, T)
            assert torch.equal(got.cpu(), want), plane
        else:
            assert torch.equal(bits(got), bits(want)), plane
    # read: the same rows back
    k2, v2 = (torch.full((N, H * 128 + 16), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tdk.tdk_kv_read(kv, cache, batch, tdk.kv_rows(k2, v2, k2.stride(0), v2.stride(0)), stream())
    torch.cuda.synchronize()
    for got, plane in ((k2, pk), (v2, pv)):
        want = torch.full(got.shape, 5.0, dtype=torch.bfloat16)
        full = plane.cpu() if fmt == tdk.KV_BF16 else bf(kh.from4(*kh.unpack4(plane.cpu(), T)))
        for r, (s, p) in enumerate(where):
            slot = b.slot(s, p) if p >= 0 else None
            want[r, :H * 128] = 0 if slot is None else full[slot].reshape(-1)
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got.float()), torch.nan_to_num(want.float()))
    return b


@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4])
@pytest.mark.parametrize("H,Hq,T,interleaved,theta,fused,pad", [(8, 40, 16, False, 1e6, True, 0), (1, 1, 16, True, 1e4, False, 3), (3, 21, 32, False, 5e5, True, 1),
                                                               (4, 28, 32, True, 1e6, True, 0), (8, 8, 16, True, 5e5, False, 2), (5, 5, 16, False, 1e4, False, 0)])
def test_append_and_read(fmt, H, Hq, T, interleaved, theta, fused, pad):
    check_append(fmt, H, Hq, T, interleaved, theta, RAGGED, fused=fused, pad=pad)


@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4])
def test_append_far_positions_and_many_sequences(fmt):
    """More sequences than one round of the search probes, positions up to 70000; one token each."""
    rng = np.random.default_rng(3)
    check_append(fmt, 2, 4, 16, False, 1e6, [(int(h), 1) for h in rng.integers(0, 70000, 3)] + [(int(h), int(n)) for h, n in zip(rng.integers(0, 40, 130), rng.integers(0, 3, 130))])


def test_append_many_tokens_take_a_wavefront_each():
    check_append(tdk.KV_BF16, 8, 16, 16, False, 1e6, [(5, 700), (0, 333)], fused=True)
    check_append(tdk.KV_MXFP4, 8, 16, 32, True, 1e6, [(5, 700), (0, 333)], fused=True)


@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4])
def test_append_skips_pages_that_are_not_there(fmt):
    def spoil(b):
        b.table[2, 1] = -1
        b.table[3, 1] = b.pool_pages
        b.table[4, 6] = 2 ** 31 - 1
        b.lens[5] = 1               # two tokens announced, one long: the first has no position
        b.lengths = list(b.lengths)
        b.lengths[5] = (-1, 2)
        b.lens[0], b.lengths[0] = 16 * b.stride + 1, (16 * b.stride, 1)          # past the table
    check_append(fmt, 2, 2, 16, False, 1e6, [(0, 1), (37, 0), (15, 18), (16, 16), (100, 3), (0, 2)], spoil=spoil)


def test_four_bits_of_unusual_values():
    def values(x):
        x[0, :32] = 0.0
        x[0, 32:64] = -0.0
        x[1, 5], x[1, 40], x[2, 70] = math.inf, -math.inf, math.nan
        x[3] = 3.0e38
        x[4] = 1e-39
        x[5, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4)      # ties
        x[6, :32] = 7.0
        x[7, :32], x[7, 0] = 1.0, 6.96875
    check_append(tdk.KV_MXFP4, 2, 2, 16, False, 1e6, [(0, 1)] + [(0, 16)], values=values)


def test_queries_rotate_in_place_and_may_be_left_out():
    H, Hq, T = 8, 8, 16
    b = kh.Batch([(40, 3), (7, 5)], T, 4)
    x = bf(torch.randn(b.n, Hq * 128, generator=torch.Generator().manual_seed(1))).cuda()
    k, v = x.clone(), x.clone()
    kv, (pk, pv) = handle(tdk.KV_BF16, H, T), pools(tdk.KV_BF16, b.pool_pages, H, T, 0.0)
    cache, batch = tdk.kv_cache(pk, pv, b.pool_pages), b.struct(tdk)
    tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(k, v, 1024, 1024), stream())
    first = [p.clone() for p in (pk, pv)]
    want = bf(kh.rotate(x.float().cpu().numpy().reshape(b.n, Hq, 128), [p for _, p in b.positions()], 1e6, False)).reshape(b.n, -1)
    tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(k, v, 1024, 1024, q=x, q_stride=1024, n_q_heads=Hq, q_out=x, q_out_stride=1024), stream())
    torch.cuda.synchronize()
    assert torch.equal(bits(x), bits(want)) and all(torch.equal(bits(a), bits(c)) for a, c in zip(first, (pk, pv)))


# ---- attention ----

def check_attend(fmt, H, group, T, lengths, window=0, sink=0, hole=None, join=False, scale=1 / math.sqrt(128), seed=1, spoil=None, poison=None, pad=0,
                 max_len=None, q_pad=0, no_lse=False, spread=2.0, extra_stride=1):
    g = torch.Generator().manual_seed(seed)
    b = kh.Batch(lengths, T, seed, pad_tokens=pad, extra_stride=extra_stride)
    Hq, N = H * group, b.n_tokens
    k, v = (bf(torch.randn(b.pool_pages, T, H, 128, generator=g)) for _ in range(2))
    if poison:
        poison(b, k, v)
    if spoil:
        spoil(b)
    if fmt == tdk.KV_MXFP4:
        dk, dv = (kh.pack4(*kh.to4(x.float()), T) for x in (k, v))
        k, v = (kh.from4(*kh.unpack4(x, T)) for x in (dk, dv))
    else:
        dk, dv = k, v
    q = bf(spread * torch.randn(N, Hq, 128, generator=g))
    part = [None, None]
    if join:
        part = [torch.randn(N, Hq, 128, generator=g), torch.randn(N, Hq, generator=g) + 3]
        part[1][::3, ::2] = -math.inf
        part[0][0, 0] = math.nan                       # of an empty part nothing is read
    want, wlse, mass, big = kh.attend(b, k.double(), v.double(), q[:b.n].double(), scale, window, sink, hole,
                                      *(None if p is None else p[:b.n].double() for p in part))
    kv = handle(fmt, H, T)
    qd = torch.zeros(N, Hq * 128 + q_pad, dtype=torch.bfloat16, device="cuda")
    qd[:, :Hq * 128] = q.reshape(N, -1).cuda()
    out = torch.full((N, Hq * 128 + q_pad), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((N, Hq), 9.0, device="cuda")
    dk, dv = dk.cuda(), dv.cuda()
    parts = [None if p is None else p.cuda() for p in part]
    hd = None if hole is None else torch.tensor(hole, dtype=torch.int32, device="cuda")
    batch = b.struct(tdk, max_len)
    need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, Hq)
    space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN wherever it is read as a number)
    io = tdk.kv_attend_io(qd, qd.stride(0), Hq, scale, out, out.stride(0), None if no_lse else lse, space, need, window, sink, hd, *parts)
    tdk.tdk_kv_attend(kv, tdk.kv_cache(dk, dv, b.pool_pages), batch, io, stream())
    torch.cuda.synchronize()
    assert (space[need:] == 0xFF).all()
    got, glse = out[:, :Hq * 128].reshape(N, Hq, 128).cpu().double(), lse.cpu().double()
    assert (out[:, Hq * 128:] == 9.0).all()
    assert (got[b.n:] == 9.0).all() and (glse[b.n:] == 9.0).all()
    got, glse = got[:b.n], glse[:b.n]
    tol, ltol = kh.tolerance(want, wlse, mass, big, max([1] + [h + n for h, n in lengths]))
    far = lambda a, c, t: int((~((a - c).abs() <= t).logical_or(a == c).logical_or(torch.isnan(a) & torch.isnan(c))).sum())      # noqa: E731
    wrong = far(got, want, torch.nan_to_num(tol, nan=0.0))
    assert wrong == 0, (wrong, got.numel(), float(torch.nan_to_num((got - want).abs() - tol).max()))
    if no_lse:
        assert (glse == 9.0).all()
    else:
        wrong = far(glse, wlse, torch.nan_to_num(ltol, nan=0.0, posinf=0.0))
        assert wrong == 0, (wrong, glse.numel(), float(torch.nan_to_num((glse - wlse).abs()).max()))
    return out, lse


FORMATS = pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4], ids=["bf16", "mxfp4"])


@FORMATS
@pytest.mark.parametrize("T", [16, 32])
@pytest.mark.parametrize("H,group", [(8, 5), (1, 16), (2, 1), (3, 7), (4, 8)])
def test_one_token_per_sequence(fmt, T, H, group):
    check_attend(fmt, H, group, T, [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (31, 1), (32, 1), (33, 1), (63, 1), (64, 1), (200, 1), (777, 1)])


@FORMATS
@pytest.mark.parametrize("T", [16, 32])
@pytest.mark.parametrize("H,group,lengths", [(2, 5, [(10, 4), (0, 3), (37, 0), (100, 2), (0, 1)]), (8, 1, [(5, 7), (16, 16), (0, 5)]),
                                             (1, 8, [(0, 40), (33, 50)]), (2, 4, [(0, 131), (70, 66), (5, 1)]), (1, 3, [(0, 300)]),
                                             (2, 8, [(300, 8), (40, 8)]), (3, 16, [(100, 1), (31, 1), (0, 1)]), (2, 16, [(90, 2), (3, 3), (50, 0)]), (8, 5, [(600, 7), (0, 7)])])
def test_several_tokens_per_sequence(fmt, T, H, group, lengths):
    check_attend(fmt, H, group, T, lengths, pad=2, q_pad=8)


@FORMATS
@pytest.mark.parametrize("T,group,lengths,kw", [(16, 33, [(70, 1), (0, 1), (300, 1)], {}), (32, 129, [(40, 1), (90, 2), (5, 0)], dict(window=20, sink=3)),
                                                (16, 300, [(130, 1), (0, 3)], dict(hole=[(30, 60), (1, 2)], join=True)), (32, 64, [(4000, 1)], {}),
                                                (16, 160, [(3000, 2)], dict(window=1500, sink=1))])
def test_more_query_heads_than_a_block_of_rows_holds(fmt, T, group, lengths, kw):
    """One KV head for all queries: a token's heads fill several blocks, or a block not quite."""
    check_attend(fmt, 1, group, T, lengths, q_pad=8, **kw)


@FORMATS
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (7, 0), (16, 4), (33, 40), (64, 1), (1000, 5), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
@pytest.mark.parametrize("lengths", [[(0, 1), (3, 1), (40, 1), (250, 1)], [(0, 70), (90, 40), (7, 3)]])
def test_windows_and_sinks(fmt, window, sink, lengths):
    check_attend(fmt, 2, 3, 16, lengths, window=window, sink=sink)


@FORMATS
@pytest.mark.parametrize("hole", [[(0, 0), (5, 5), (0, 32)], [(0, 1000), (32, 64), (1, 250)], [(3, 2), (-5, 17), (17, 2 ** 31 - 1)],
                                  [(-2 ** 31, 5), (-2 ** 31, 2 ** 31 - 1), (2 ** 31 - 1, -2 ** 31)]])
@pytest.mark.parametrize("lengths", [[(0, 1), (90, 1), (250, 1)], [(8, 40), (64, 3), (250, 20)]])
@pytest.mark.parametrize("window,sink,join", [(0, 0, False), (0, 0, True), (40, 20, True)])
def test_holes_and_joined_parts(fmt, hole, lengths, window, sink, join):
    """Among them queries that see nothing at all, with and without a part to join."""
    check_attend(fmt, 2, 2, 16, lengths, window=window, sink=sink, hole=hole, join=join)


@FORMATS
@pytest.mark.parametrize("scale", [0.0, -0.0, -0.1, 1.0, 3e-39])
def test_scales(fmt, scale):
    check_attend(fmt, 2, 4, 16, [(50, 1), (20, 12)], scale=scale)


@FORMATS
@pytest.mark.parametrize("lengths", [[(5000, 1)], [(3000, 1), (10, 1)], [(2500, 9)]])
@pytest.mark.parametrize("max_len", [None, 1, 100000])
def test_long_sequences_are_cut_and_joined(fmt, lengths, max_len):
    check_attend(fmt, 2, 5, 16, lengths, max_len=max_len, join=True)


@FORMATS
def test_long_window(fmt):
    check_attend(fmt, 1, 4, 32, [(4000, 1), (2000, 3)], window=1500, sink=4)


@FORMATS
def test_pages_that_are_not_there_are_not_seen(fmt):
    def spoil(b):
        b.table[0, 1], b.table[1, 0], b.table[2, 3] = -1, b.pool_pages, -2 ** 31
        b.lens[3], b.lengths = 16 * b.stride + 40, [*b.lengths[:3], (16 * b.stride + 39, 1)]          # longer than its table
    check_attend(fmt, 2, 4, 16, [(50, 1), (20, 12), (60, 40), (30, 1)], spoil=spoil)


@FORMATS
@pytest.mark.parametrize("lengths", [[(50, 1), (200, 1)], [(50, 20), (10, 70), (0, 3)]])
def test_what_is_not_seen_may_hold_anything(fmt, lengths):
    """Rows behind the end, in pages of nobody, and behind the window: NaN and infinities.  A window of 8 and one sink."""
    def poison(b, k, v):
        used = {b.slot(s, j) for s, (h, n) in enumerate(b.lengths) for p in range(h, h + n) for j in range(p + 1) if j == 0 or j > p - 8}
        for pg in range(b.pool_pages):
            for t in range(b.T):
                if (pg, t) not in used:
                    k[pg, t], v[pg, t] = (math.nan, math.inf) if t & 1 else (-math.inf, math.nan)
    check_attend(fmt, 2, 3, 16, lengths, window=8, sink=1, poison=poison)


@FORMATS
@pytest.mark.parametrize("lengths,group", [([(30, 40)], 3), ([(0, 4)], 4), ([(3, 150)], 2)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(fmt, lengths, group):
    """One token's V is infinite in some elements, another's NaN: queries before them stay finite, queries behind do not."""
    def poison(b, k, v):
        h, n = b.lengths[0]
        v[b.slot(0, h + 1)][:, 32:40] = math.inf
        v[b.slot(0, h + n // 2)][:, 100] = math.nan
    out, _ = check_attend(fmt, 2, group, 16, lengths, poison=poison)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[-1]).any()


@FORMATS
@pytest.mark.parametrize("lengths", [[(40, 1)], [(20, 30)], [(600, 1)]])
def test_keys_that_are_not_finite(fmt, lengths):
    def poison(b, k, v):
        k[b.slot(0, 18)][0] = math.nan
    check_attend(fmt, 2, 2, 16, lengths, poison=poison)


def test_without_lse_and_nothing_to_do():
    check_attend(tdk.KV_BF16, 2, 2, 16, [(9, 3)], no_lse=True)
    check_attend(tdk.KV_BF16, 2, 2, 16, [(9, 0), (0, 0), (5, 1)], pad=4)
    check_attend(tdk.KV_BF16, 1, 1, 16, [(3, 1)] * 200)


def test_weights_far_apart():
    """Scores over some hundred: one token's weight is all there is, and the reference point moves often."""
    check_attend(tdk.KV_BF16, 2, 4, 16, [(300, 1), (100, 30)], spread=40.0, scale=0.5)
