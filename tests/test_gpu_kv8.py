"""Paged caches in 8 bits on the GPU: unusual values bit for bit, and attention over the pages against plain forms in 64 bits, by tolerances that
follow from its arithmetic (kv_helpers.tolerance)."""
import math

import numpy as np
import pytest
import torch

import kv_helpers as kh
import rope_helpers as rh
from paper_2604_03143_amd import tdk
from test_gpu_rope import PLAIN, check_append

pytestmark = pytest.mark.gpu
FMT = tdk.KV_MXFP8


def stream():
    return torch.cuda.current_stream().cuda_stream


def bf(x):
    return torch.as_tensor(x).to(torch.bfloat16)


def test_eight_bits_of_unusual_values():
    ties = torch.tensor([0.0009765625, 0.0029296875, 17.0, 19.0, 464.0, 432.0, 240.0, 448.0])

    def values(x):
        x[0, :32] = 0.0
        x[0, 32:64] = -0.0
        x[1, 5], x[1, 40], x[2, 70] = math.inf, -math.inf, math.nan
        x[3] = 3.0e38
        x[4] = 1e-39
        x[5, :32] = torch.cat([ties] * 4)
        x[6, :32], x[6, 0] = 1.0, 466.0
        x[7, :32], x[7, 0] = 2.0 ** -9, 464.0
        x[8, :32] = torch.cat([ties] * 4) * 2.0 ** -126
        x[9, :32] = 2.0 ** 127 * 1.8125                # (what a byte of 246 holds, and the next power from just above)
        x[10, :32] = 2.0 ** 127 * 1.8203125
        x[10, 1:8] = 2.0 ** 127 * 1.5
    check_append(FMT, 2, 2, 16, 1e6, False, 128, PLAIN, [(0, 1)] + [(0, 16)], values=values)


def test_every_code_and_power_is_read_as_bf16_has_it():
    """Pages written by hand: all 256 bytes under all 256 powers of two."""
    T, H, pages = 16, 1, 32
    code = torch.arange(256, dtype=torch.uint8).reshape(2, 128).repeat(256, 1).reshape(pages, T, H, 128)
    byte = torch.arange(256, dtype=torch.uint8).repeat_interleave(2)[:, None].expand(512, 4).reshape(pages, T, H, 4)
    pool = rh.pack8(code, byte, T).cuda()
    b = kh.Batch([(0, 512)], T, 1, spare=0)
    b.table[0, :pages] = np.arange(pages)
    kv, batch = tdk.tdk_kv_create(tdk.model(1, H, 128, T), FMT), b.struct(tdk)
    k, v = (torch.zeros(512, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tdk.tdk_kv_read(kv, tdk.kv_cache(pool, pool, pages), batch, tdk.kv_rows(k, v, 128, 128), stream())
    torch.cuda.synchronize()
    want = bf(rh.from8(code, byte)).reshape(512, 128)
    for got in (k.cpu(), v.cpu()):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.where(torch.isnan(got), torch.zeros_like(got), got), torch.where(torch.isnan(want), torch.zeros_like(want), want))


# ---- attention ----

def check_attend(H, group, T, lengths, window=0, sink=0, hole=None, join=False, scale=1 / math.sqrt(128), seed=1, spoil=None, poison=None, pad=0,
                 max_len=None, q_pad=0, no_lse=False, spread=2.0, extra_stride=1, raw=None):
    g = torch.Generator().manual_seed(seed)
    b = kh.Batch(lengths, T, seed, pad_tokens=pad, extra_stride=extra_stride)
    Hq, N = H * group, b.n_tokens
    k, v = (bf(torch.randn(b.pool_pages, T, H, 128, generator=g)) for _ in range(2))
    if poison:
        poison(b, k, v)
    if spoil:
        spoil(b)
    dk, dv = (rh.pack8(*rh.to8(x.float()), T) for x in (k, v))
    if raw:
        raw(b, dk, dv)
    k, v = (rh.from8(*rh.unpack8(x, T)) for x in (dk, dv))
    q = bf(spread * torch.randn(N, Hq, 128, generator=g))
    part = [None, None]
    if join:
        part = [torch.randn(N, Hq, 128, generator=g), torch.randn(N, Hq, generator=g) + 3]
        part[1][::3, ::2] = -math.inf
        part[0][0, 0] = math.nan                       # of an empty part nothing is read
    want, wlse, mass, big = kh.attend(b, k, v, q[:b.n].double(), scale, window, sink, hole, *(None if p is None else p[:b.n].double() for p in part))
    kv = tdk.tdk_kv_create(tdk.model(1, H, 128, T), FMT)
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


@pytest.mark.parametrize("T", [16, 32])
@pytest.mark.parametrize("H,group", [(8, 5), (1, 16), (2, 1), (3, 7), (4, 8)])
def test_one_token_per_sequence(T, H, group):
    check_attend(H, group, T, [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (31, 1), (32, 1), (33, 1), (63, 1), (64, 1), (200, 1), (777, 1)])


@pytest.mark.parametrize("T", [16, 32])
@pytest.mark.parametrize("H,group,lengths", [(2, 5, [(10, 4), (0, 3), (37, 0), (100, 2), (0, 1)]), (8, 1, [(5, 7), (16, 16), (0, 5)]),
                                             (1, 8, [(0, 40), (33, 50)]), (2, 4, [(0, 131), (70, 66), (5, 1)]), (1, 3, [(0, 300)]),
                                             (2, 8, [(300, 8), (40, 8)]), (3, 16, [(100, 1), (31, 1), (0, 1)]), (2, 16, [(90, 2), (3, 3), (50, 0)]), (8, 5, [(600, 7), (0, 7)])])
def test_several_tokens_per_sequence(T, H, group, lengths):
    check_attend(H, group, T, lengths, pad=2, q_pad=8)


@pytest.mark.parametrize("T,group,lengths,kw", [(16, 33, [(70, 1), (0, 1), (300, 1)], {}), (32, 129, [(40, 1), (90, 2), (5, 0)], dict(window=20, sink=3)),
                                                (16, 300, [(130, 1), (0, 3)], dict(hole=[(30, 60), (1, 2)], join=True)), (32, 64, [(4000, 1)], {}),
                                                (16, 160, [(3000, 2)], dict(window=1500, sink=1))])
def test_more_query_heads_than_a_block_of_rows_holds(T, group, lengths, kw):
    check_attend(1, group, T, lengths, q_pad=8, **kw)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (7, 0), (16, 4), (33, 40), (64, 1), (1000, 5), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
@pytest.mark.parametrize("lengths", [[(0, 1), (3, 1), (40, 1), (250, 1)], [(0, 70), (90, 40), (7, 3)], [(60, 6), (200, 6)]])
def test_windows_and_sinks(window, sink, lengths):
    check_attend(2, 3, 16, lengths, window=window, sink=sink)


@pytest.mark.parametrize("hole", [[(0, 0), (5, 5), (0, 32)], [(0, 1000), (32, 64), (1, 250)], [(3, 2), (-5, 17), (17, 2 ** 31 - 1)],
                                  [(-2 ** 31, 5), (-2 ** 31, 2 ** 31 - 1), (2 ** 31 - 1, -2 ** 31)]])
@pytest.mark.parametrize("lengths", [[(0, 1), (90, 1), (250, 1)], [(8, 40), (64, 3), (250, 20)]])
@pytest.mark.parametrize("window,sink,join", [(0, 0, False), (0, 0, True), (40, 20, True)])
def test_holes_and_joined_parts(hole, lengths, window, sink, join):
    """Among them queries that see nothing at all, with and without a part to join."""
    check_attend(2, 2, 16, lengths, window=window, sink=sink, hole=hole, join=join)


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.1, 1.0, 3e-39])
def test_scales(scale):
    check_attend(2, 4, 16, [(50, 1), (20, 12)], scale=scale)


@pytest.mark.parametrize("lengths", [[(5000, 1)], [(3000, 1), (10, 1)], [(2500, 9)]])
@pytest.mark.parametrize("max_len", [None, 1, 100000])
def test_long_sequences_are_cut_and_joined(lengths, max_len):
    check_attend(2, 5, 16, lengths, max_len=max_len, join=True)


def test_long_window():
    check_attend(1, 4, 32, [(4000, 1), (2000, 3)], window=1500, sink=4)


def test_pages_that_are_not_there_are_not_seen():
    def spoil(b):
        b.table[0, 1], b.table[1, 0], b.table[2, 3] = -1, b.pool_pages, -2 ** 31
        b.lens[3], b.lengths = 16 * b.stride + 40, [*b.lengths[:3], (16 * b.stride + 39, 1)]          # longer than its table
    check_attend(2, 4, 16, [(50, 1), (20, 12), (60, 40), (30, 1)], spoil=spoil)


@pytest.mark.parametrize("lengths", [[(50, 1), (200, 1)], [(50, 20), (10, 70), (0, 3)], [(50, 6), (200, 6)]])
@pytest.mark.parametrize("how", ["values", "codes", "powers"])
def test_what_is_not_seen_may_hold_anything(lengths, how):
    """Rows behind the end, in pages of nobody, and behind the window: NaN and infinities, as blocks, as single bytes, as powers beyond bf16's range.  A
    window of 8 and one sink."""
    def unused(b):
        used = {b.slot(s, j) for s, (h, n) in enumerate(b.lengths) for p in range(h, h + n) for j in range(p + 1) if j == 0 or j > p - 8}
        return [(pg, t) for pg in range(b.pool_pages) for t in range(b.T) if (pg, t) not in used]

    def poison(b, k, v):
        for pg, t in unused(b):
            k[pg, t], v[pg, t] = (math.nan, math.inf) if t & 1 else (-math.inf, math.nan)

    def raw(b, dk, dv):
        for pg, t in unused(b):
            for x in (dk, dv):
                if how == "codes":
                    x[pg, :, 128 * t + 5], x[pg, :, 128 * t + 77] = 0x7F, 0xFF
                else:
                    x[pg, :, 128 * b.T + 4 * t:128 * b.T + 4 * t + 4] = torch.tensor([254, 255, 250, 247], dtype=torch.uint8)
    check_attend(2, 3, 16, lengths, window=8, sink=1, **(dict(poison=poison) if how == "values" else dict(raw=raw)))


@pytest.mark.parametrize("lengths,group", [([(30, 40)], 3), ([(0, 4)], 4), ([(3, 150)], 2), ([(9, 10)], 3)])
@pytest.mark.parametrize("how", ["blocks", "codes"])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(lengths, group, how):
    """One token's V is NaN in a block, another's in one element, and infinite in another: queries before them stay finite, queries behind do not."""
    def raw(b, dk, dv):
        h, n = b.lengths[0]
        pg, t = b.slot(0, h + 1)
        if how == "blocks":
            dv[pg, :, 128 * b.T + 4 * t + 1] = 255
        else:
            dv[pg, :, 128 * t + 33] = 0x7F
        pg, t = b.slot(0, h + n // 2)
        dv[pg, :, 128 * b.T + 4 * t + 2] = 247         # 2^120
        dv[pg, :, 128 * t + 64:128 * t + 96] = 0x30
        dv[pg, :, 128 * t + 70] = 0x7E                 # 448: infinite
        dv[pg, :, 128 * t + 71] = 0xFE
    out, _ = check_attend(2, group, 16, lengths, raw=raw)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[-1]).any() and torch.isinf(out[-1]).any()


@pytest.mark.parametrize("lengths", [[(40, 1)], [(20, 30)], [(600, 1)], [(30, 9)]])
def test_keys_that_are_not_finite(lengths):
    def raw(b, dk, dv):
        pg, t = b.slot(0, 18)
        dk[pg, 0, 128 * t + 3] = 0x7F
        dk[pg, 1, 128 * b.T + 4 * t + 3] = 255
    check_attend(2, 2, 16, lengths, raw=raw)


@pytest.mark.parametrize("lengths", [[(40, 1)], [(20, 30)], [(30, 9)]])
@pytest.mark.parametrize("size", [1e-30, 1e33])
def test_values_of_other_sizes(lengths, size):
    """V far from one: weights are one at most, so sums of values of 1e33 stay finite, and those of 1e-30 keep their places."""
    def poison(b, k, v):
        v.mul_(size)
    check_attend(2, 2, 16, lengths, poison=poison)


def test_no_lse_and_queries_of_no_sequence():
    check_attend(2, 2, 16, [(40, 1), (0, 0), (3, 2)], no_lse=True, pad=5)
    check_attend(2, 2, 16, [(0, 0), (0, 0)], pad=3)


@pytest.mark.parametrize("seed", range(6))
def test_random_batches(seed):
    rng = np.random.default_rng(seed)
    H, T = int(rng.choice([1, 2, 3, 8])), int(rng.choice([16, 32]))
    group = int(rng.choice([1, 2, 4, 5, 7, 8, 16]))
    lengths = [(int(rng.integers(0, 400)), int(rng.choice([0, 1, 2, int(rng.integers(1, 60))]))) for _ in range(int(rng.integers(1, 12)))]
    kw = {}
    if rng.random() < 0.5:
        kw = dict(window=int(rng.integers(1, 200)), sink=int(rng.integers(0, 20)))
    if rng.random() < 0.5:
        kw.update(hole=[tuple(sorted(rng.integers(0, 400, 2).tolist())) for _ in lengths], join=bool(rng.random() < 0.7))
    check_attend(H, group, T, lengths, seed=seed, pad=int(rng.integers(0, 4)), q_pad=8 * int(rng.integers(0, 3)), **kw)
