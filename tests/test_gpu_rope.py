"""Rotation by scaled frequencies and of part of the head on the GPU, bit for bit: tdk_kv_rotate, tdk_kv_append and the rounds' calls."""
import math

import numpy as np
import pytest
import torch

import kv_helpers as kh
import rope_helpers as rh
from paper_2604_03143_amd import tdk

pytestmark = pytest.mark.gpu
SCALINGS = {"none": tdk.ROPE_SCALE_NONE, "linear": tdk.ROPE_SCALE_LINEAR, "turns": tdk.ROPE_SCALE_TURNS, "index": tdk.ROPE_SCALE_INDEX}
PLAIN = dict(scaling="none")
LINEAR = dict(scaling="linear", factor=4.0)
TURNS = dict(scaling="turns", factor=8.0, original=8192, low=1.0, high=4.0)
INDEX = dict(scaling="index", factor=32.0, original=4096, low=1.0, high=32.0, magnitude=0.1 * math.log(32.0) + 1.0)
# lengths: (earlier tokens, new tokens) per sequence
RAGGED = [(0, 1), (37, 0), (15, 18), (16, 16), (100000, 3), (1, 1)]


def stream():
    return torch.cuda.current_stream().cuda_stream


def bf(x):
    return torch.as_tensor(x).to(torch.bfloat16)


def bits(t):
    return t.contiguous().view(torch.int16).cpu()


def handle(fmt, H, T, theta, interleaved, rotary, s):
    model = tdk.model(1, H, 128, T, theta, tdk.ROPE_INTERLEAVED if interleaved else tdk.ROPE_HALF)
    rope = tdk.rope(rotary, SCALINGS[s["scaling"]], s.get("factor", 1.0), s.get("original", 0), s.get("low", 0), s.get("high", 0), s.get("magnitude", 1.0))
    return tdk.tdk_kv_create_rope(model, rope, fmt)


def expected(x, pos, theta, interleaved, rotary, s, back=False):
    return rh.rotate(x, pos, rh.frequencies(theta, rotary, **s), rotary, interleaved, s.get("magnitude", 1.0), back)


def check_rotate(H, Hq, theta, interleaved, rotary, s, lengths, back=False, planes="kq", pad=0, in_place=False, fused=False, seed=1, spoil=None):
    g = torch.Generator().manual_seed(seed)
    b = kh.Batch(lengths, 16, seed, pad_tokens=pad)
    if spoil:
        spoil(b)
    N = b.n_tokens
    x = bf(torch.randn(N, (Hq + H) * 128 + 8, generator=g))
    if fused:
        xd = x.cuda()
        q, k = xd[:, :Hq * 128], xd[:, Hq * 128:(Hq + H) * 128]
    else:
        q, k = x[:, :Hq * 128].contiguous().cuda(), x[:, Hq * 128:(Hq + H) * 128].contiguous().cuda()
    outs = {}
    for name, src, heads in (("k", k, H), ("q", q, Hq)):
        outs[name] = src if in_place else torch.full((N, heads * 128 + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    kv = handle(tdk.KV_BF16, H, 16, theta, interleaved, rotary, s)
    batch = b.struct(tdk)
    batch.block_table, batch.table_stride = None, 0
    kw = {}
    if "q" in planes:
        kw = dict(q=q, q_stride=q.stride(0), n_q_heads=Hq, q_out=outs["q"], q_out_stride=outs["q"].stride(0))
    kk = (k, k.stride(0), outs["k"], outs["k"].stride(0)) if "k" in planes else (None, 0, None, 0)
    tdk.tdk_kv_rotate(kv, batch, tdk.kv_rotate_io(*kk, **kw, back=back), stream())
    torch.cuda.synchronize()
    pos = [p for _, p in b.positions()]
    keep = [i for i, p in enumerate(pos) if p >= 0]
    xf = x.float().numpy()
    for name, heads, cols in (("k", H, slice(Hq * 128, (Hq + H) * 128)), ("q", Hq, slice(0, Hq * 128))):
        old = x[:, cols] if in_place else torch.full((N, heads * 128), 3.0, dtype=torch.bfloat16)
        want = old.clone()
        if name in planes and keep:
            rows = xf[keep][:, cols].reshape(len(keep), heads, 128)
            want[keep] = bf(expected(rows, [pos[i] for i in keep], theta, interleaved, rotary, s, back)).reshape(len(keep), -1)
        assert torch.equal(bits(outs[name][:, :heads * 128]), bits(want)), name
        if not in_place:
            assert (outs[name][:, heads * 128:] == 3.0).all()


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rotary", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("s", [PLAIN, LINEAR, TURNS, INDEX], ids=lambda s: s["scaling"])
def test_rotate(interleaved, rotary, s):
    check_rotate(3, 6, 5e5, interleaved, rotary, s, RAGGED, pad=2)


@pytest.mark.parametrize("interleaved,rotary,s", [(False, 128, TURNS), (True, 64, INDEX), (False, 96, INDEX), (True, 128, PLAIN), (False, 32, LINEAR)])
@pytest.mark.parametrize("kw", [dict(back=True), dict(in_place=True), dict(in_place=True, back=True, fused=True), dict(planes="k"), dict(planes="q"), dict(fused=True, pad=3)],
                         ids=lambda kw: "-".join(kw))
def test_rotate_back_in_place_one_plane_and_slices(interleaved, rotary, s, kw):
    check_rotate(8, 40, 1e6, interleaved, rotary, s, RAGGED, **kw)


@pytest.mark.parametrize("H,Hq", [(1, 1), (5, 35), (8, 128), (2, 2)])
@pytest.mark.parametrize("lengths", [[(5, 700), (0, 333)], [(0, 1)], [(2 ** 21, 5)]])
@pytest.mark.parametrize("interleaved,rotary", [(False, 64), (True, 128)])
def test_rotate_many_tokens_and_head_counts(H, Hq, lengths, interleaved, rotary):
    check_rotate(H, Hq, 1e4, interleaved, rotary, TURNS, lengths, fused=True)


@pytest.mark.parametrize("H,Hq", [(1, 1), (4, 4), (4, 10), (8, 16), (3, 28), (8, 33)])
@pytest.mark.parametrize("interleaved,rotary", [(False, 16), (False, 112), (False, 128), (True, 48)])
def test_rotate_many_tokens_with_one_wavefront_each_to_four(H, Hq, interleaved, rotary):
    check_rotate(H, Hq, 1e4, interleaved, rotary, TURNS, [(7, 1300), (0, 1), (2, 900)], pad=1)
    check_rotate(H, Hq, 1e4, interleaved, rotary, TURNS, [(7, 1300), (2, 900)], in_place=True, fused=True)


def test_rotate_leaves_tokens_without_a_position_alone():
    def spoil(b):
        b.lens[1] = 1                 # two tokens announced, one long: the first has no position
        b.lengths = [b.lengths[0], (-1, 2), b.lengths[2]]
    check_rotate(2, 4, 1e6, False, 64, TURNS, [(3, 2), (0, 2), (9, 1)], spoil=spoil, pad=1)
    check_rotate(2, 4, 1e6, False, 64, TURNS, [(3, 0), (0, 0)], pad=4)


def test_values_that_are_not_finite_stay_in_their_pair():
    H, b = 2, kh.Batch([(10, 2)], 16, 1)
    x = torch.ones(2, H * 128)
    x[0, 3], x[0, 100], x[1, 128 + 64] = math.inf, math.nan, -math.inf
    for interleaved in (False, True):
        k = bf(x).cuda()
        batch = b.struct(tdk)
        out = torch.zeros_like(k)
        tdk.tdk_kv_rotate(handle(tdk.KV_BF16, H, 16, 1e6, interleaved, 64, TURNS), batch, tdk.kv_rotate_io(k, 256, out, 256), stream())
        torch.cuda.synchronize()
        got = out.cpu().float()
        pair = 2 if interleaved else 35
        odd = {(0, 3), (0, pair), (0, 100), (1, 192)}
        assert {tuple(i) for i in (~torch.isfinite(got)).nonzero().tolist()} == odd
        assert torch.isnan(got[0, 100]) and got[1, 192] == -math.inf


def test_far_positions_turned_there_and_back():
    """Rows at two million tokens, turned there in one call and back in another: two roundings to bf16, 2^-8 of the pair's length each, and twice the
    products' 2^-24."""
    H, b = 4, kh.Batch([(2 * 10 ** 6, 50)], 16, 1, extra_stride=0)
    k = bf(torch.randn(50, H * 128, generator=torch.Generator().manual_seed(3))).cuda()
    mid, end = torch.zeros_like(k), torch.zeros_like(k)
    kv, batch = handle(tdk.KV_BF16, H, 16, 5e5, False, 128, INDEX), b.struct(tdk)
    tdk.tdk_kv_rotate(kv, batch, tdk.kv_rotate_io(k, H * 128, mid, H * 128), stream())
    tdk.tdk_kv_rotate(kv, batch, tdk.kv_rotate_io(mid, H * 128, end, H * 128, back=True), stream())
    torch.cuda.synchronize()
    x, y = (t.cpu().double().reshape(50, H, 2, 64) for t in (k, end))
    size = x.norm(dim=2, keepdim=True)
    assert not torch.equal(mid, k) and ((x - y).abs() <= (2.0 ** -8 * (1 + math.sqrt(2)) * 1.01 + 2.0 ** -20) * size).all()


# ---- the append with the same frequencies ----

def check_append(fmt, H, Hq, T, theta, interleaved, rotary, s, lengths, fused=False, pad=0, seed=1, values=None, spoil=None):
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
    q, k, v = parts if fused else [p.contiguous() for p in parts]
    kv = handle(fmt, H, T, theta, interleaved, rotary, s)
    size = tdk.tdk_kv_page_bytes(kv)
    pk, pv = (torch.full((b.pool_pages, size), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2))
    q_out = torch.full((N, Hq * 128 + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    batch, cache = b.struct(tdk), tdk.kv_cache(pk, pv, b.pool_pages)
    rows = tdk.kv_rows(k, v, k.stride(0), v.stride(0), q=q, q_stride=q.stride(0), n_q_heads=Hq, q_out=q_out, q_out_stride=q_out.stride(0))
    tdk.tdk_kv_append(kv, cache, batch, rows, stream())
    torch.cuda.synchronize()
    where = b.positions()
    n, pos = len(where), [p for _, p in where]
    xf = x.float().numpy()
    want_q = bf(expected(xf[:n, :Hq * 128].reshape(n, Hq, 128), pos, theta, interleaved, rotary, s))
    kr = expected(xf[:n, Hq * 128:(Hq + H) * 128].reshape(n, H, 128), pos, theta, interleaved, rotary, s)
    vr = x[:n, (Hq + H) * 128:].reshape(n, H, 128)
    seen = [i for i, p in enumerate(pos) if p >= 0]
    left = [i for i in range(N) if i not in set(seen)]
    assert torch.equal(bits(q_out[seen, :Hq * 128]), bits(want_q[seen].reshape(len(seen), -1)))
    assert (q_out[left] == 3.0).all() and (q_out[:, Hq * 128:] == 3.0).all()
    old = torch.full((b.pool_pages, size), 0x5A, dtype=torch.uint8)
    full = []
    for plane, (got, new) in enumerate(((pk, torch.as_tensor(kr)), (pv, vr.float()))):
        slots = [(r, b.slot(*where[r])) for r in seen if b.slot(*where[r]) is not None]
        if fmt == tdk.KV_BF16:
            want = old.view(torch.bfloat16).reshape(b.pool_pages, T, H, 128).clone()
            for r, slot in slots:
                want[slot] = bf(kr[r]) if plane == 0 else vr[r]
            full.append(want.double())
            assert torch.equal(got.cpu(), want.view(torch.uint8).reshape(b.pool_pages, size)), plane
            continue
        four = fmt == tdk.KV_MXFP4
        code, byte = (t.clone() for t in (kh.unpack4 if four else rh.unpack8)(old.reshape(b.pool_pages, H, -1), T))
        c, e = (kh.to4 if four else rh.to8)(new)
        for r, slot in slots:
            code[slot], byte[slot] = c[r], e[r]
        assert torch.equal(got.cpu(), (kh.pack4 if four else rh.pack8)(code, byte, T).reshape(b.pool_pages, size)), plane
        full.append((kh.from4 if four else rh.from8)(code, byte))
    # read: the same rows back
    k2, v2 = (torch.full((N, H * 128 + 16), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tdk.tdk_kv_read(kv, cache, batch, tdk.kv_rows(k2, v2, k2.stride(0), v2.stride(0)), stream())
    torch.cuda.synchronize()
    for got, plane in ((k2, full[0]), (v2, full[1])):
        want = torch.full(got.shape, 5.0, dtype=torch.bfloat16)
        for r, (q_, p) in enumerate(where):
            slot = b.slot(q_, p) if p >= 0 else None
            want[r, :H * 128] = 0 if slot is None else bf(plane[slot]).reshape(-1)
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got.float(), posinf=math.inf, neginf=-math.inf), torch.nan_to_num(want.float(), posinf=math.inf, neginf=-math.inf))
    return b


SHORT = [(0, 1), (37, 0), (15, 18), (16, 16), (100, 3), (1, 1)]
ALL = pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4, tdk.KV_MXFP8], ids=["bf16", "mxfp4", "mxfp8"])


@ALL
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rotary,s", [(16, PLAIN), (32, INDEX), (48, TURNS), (64, TURNS), (80, PLAIN), (96, INDEX), (112, LINEAR), (128, TURNS), (128, INDEX), (128, LINEAR)])
def test_append_of_part_of_the_head_and_scaled(fmt, interleaved, rotary, s):
    check_append(fmt, 3, 6, 16, 5e5, interleaved, rotary, s, SHORT, pad=2)


@ALL
@pytest.mark.parametrize("H,Hq,T,fused,lengths", [(8, 40, 16, True, [(5, 700), (0, 333)]), (8, 64, 32, True, [(9, 300)]), (1, 1, 16, False, [(3, 2500)]),
                                                  (5, 5, 32, False, SHORT), (4, 28, 16, True, [(70000, 3), (0, 1)])])
def test_append_many_tokens_and_head_counts(fmt, H, Hq, T, fused, lengths):
    check_append(fmt, H, Hq, T, 1e6, False, 64, TURNS, lengths, fused=fused)
    check_append(fmt, H, Hq, T, 1e6, True, 128, INDEX, lengths, fused=fused)


def test_rounds_turn_by_the_same_frequencies():
    """Masters re-rotated into two agents' pages by a round made with the same frequencies: the library's arithmetic for the differences of positions."""
    H, T, S = 2, 16, 40
    g = torch.Generator().manual_seed(4)
    mk, mv = (bf(torch.randn(S, H, 128, generator=g)).cuda() for _ in range(2))
    pos0, tables = [21, 9000], [np.arange(5, dtype=np.int32), np.arange(568, dtype=np.int32) % 4 + 5]
    tables[1][9000 // 16:] = np.arange(568 - 9000 // 16) + 5
    pk, pv = (torch.zeros(16, T, H, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rope = tdk.rope(128, tdk.ROPE_SCALE_INDEX, 32.0, 4096, 1.0, 32.0, 1.3)
    r = tdk.tdk_round_create_rope(tdk.model(1, H, 128, T, 1e4), rope, [S], [3], [0, 0], pos0, tables)
    tdk.tdk_rerotate_round(r, 0, tdk.layer_io(mk, mv, pk, pv, 16), stream())
    torch.cuda.synchronize()
    f = rh.frequencies(1e4, 128, "index", 32.0, 4096, 1.0, 32.0)
    x = mk.cpu().float().numpy()
    for i in range(2):
        want = bf(rh.rotate(x, np.full(S, pos0[i] - 3), f, 128, False))
        for m in range(S):
            p = pos0[i] + m
            assert torch.equal(bits(pk[int(tables[i][p // T]), p % T]), bits(want[m])), (i, m)
            assert torch.equal(bits(pv[int(tables[i][p // T]), p % T]), bits(mv[m]))
    r.destroy()
