"""tdk_prompt_attend on the GPU against plain forms in 64 bits, by tolerances that follow from its arithmetic (kv_helpers.tolerance)."""
import math

import numpy as np
import pytest
import torch

import kv_helpers as kh
import prompt_helpers as ph
from paper_2604_03143_amd import tdk

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def bf(x):
    return torch.as_tensor(x).to(torch.bfloat16)


def starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)


def far(a, c, t):
    return int((~((a - c).abs() <= t).logical_or(a == c).logical_or(torch.isnan(a) & torch.isnan(c))).sum())


def check(H, group, lengths, window=0, sink=0, join=False, scale=1 / math.sqrt(128), seed=1, poison=None, pad_q=0, pad_k=0, stride_pad=0, fused=False, max_len=None,
          f32=False, no_lse=False, spread=2.0, size=1.0):
    """lengths: (queries, keys) per sequence."""
    g = torch.Generator().manual_seed(seed)
    Hq, n, m = H * group, sum(x for x, _ in lengths), sum(x for _, x in lengths)
    N, M = n + pad_q, m + pad_k
    q = bf(spread * torch.randn(N, Hq, 128, generator=g))
    k, v = bf(torch.randn(M, H, 128, generator=g)), bf(torch.randn(M, H, 128, generator=g) * size)
    if pad_k:
        k[m:], v[m:] = math.nan, math.inf
    if poison:
        poison(k, v)
    part = [None, None]
    if join:
        part = [torch.randn(N, Hq, 128, generator=g), torch.randn(N, Hq, generator=g) + 3]
        part[1][::3, ::2] = -math.inf
        part[0][0, 0] = math.nan                       # of an empty part nothing is read
    on = lambda x: x.cuda().double()       # noqa: E731  (the plain form runs on the GPU too, in 64 bits)
    want, wlse, mass, big = ph.attend(lengths, on(q[:n]), on(k[:m]), on(v[:m]), scale, window, sink, *(None if p is None else on(p[:n]) for p in part))
    want, wlse, mass = want.cpu(), wlse.cpu(), mass.cpu()
    if fused:
        assert N == M
        rows = torch.cat((q.flatten(1), k.flatten(1), v.flatten(1)), 1).cuda()
        dq, dk, dv = torch.split(rows, [Hq * 128, H * 128, H * 128], 1)
    else:
        dq, dk, dv = (torch.full((x.shape[0], x.shape[1] * 128 + stride_pad), math.nan, dtype=torch.bfloat16, device="cuda") for x in (q, k, v))
        for d, x in ((dq, q), (dk, k), (dv, v)):
            d[:, :x.shape[1] * 128] = x.flatten(1).cuda()
    out = torch.full((N, Hq * 128 + stride_pad), 9.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    lse = torch.full((N, Hq), 9.0, device="cuda")
    qs, ks = starts([x for x, _ in lengths]).cuda(), starts([x for _, x in lengths]).cuda()
    parts = [None if p is None else p.cuda() for p in part]
    kv = tdk.tdk_kv_create(tdk.model(1, H))
    batch = tdk.prompt_batch(len(lengths), N, M, max([x for _, x in lengths] + [0]) if max_len is None else max_len, qs, ks)
    need = tdk.tdk_prompt_attend_workspace_bytes(kv, batch, Hq)
    space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN wherever it is read as a number)
    io = tdk.prompt_attend_io(dq, dq.stride(0), Hq, dk, dk.stride(0), dv, dv.stride(0), scale, out, out.stride(0), None if no_lse else lse, space, need, window, sink, *parts,
                              out_f32=f32)
    tdk.tdk_prompt_attend(kv, batch, io, stream())
    torch.cuda.synchronize()
    assert (space[need:] == 0xFF).all()
    got, glse = out[:, :Hq * 128].reshape(N, Hq, 128).cpu().double(), lse.cpu().double()
    assert (out[:, Hq * 128:] == 9.0).all() and (got[n:] == 9.0).all() and (glse[n:] == 9.0).all()
    got, glse = got[:n], glse[:n]
    tol, ltol = kh.tolerance(want, wlse, mass, big, max([1] + [x for _, x in lengths]))
    wrong = far(got, want, torch.nan_to_num(tol, nan=0.0, posinf=0.0))
    assert wrong == 0, (wrong, got.numel(), float(torch.nan_to_num((got - want).abs() - tol).max()))
    if no_lse:
        assert (glse == 9.0).all()
    else:
        wrong = far(glse, wlse, torch.nan_to_num(ltol, nan=0.0, posinf=0.0))
        assert wrong == 0, (wrong, glse.numel(), float(torch.nan_to_num((glse - wlse).abs()).max()))
    return out, lse


def same(*n):
    return [(x, x) for x in n]


# enough row blocks of enough sequences that no work is split
WIDE = same(*[400] * 17)


@pytest.mark.parametrize("H,group", [(8, 5), (1, 16), (2, 1), (3, 7), (4, 8)])
@pytest.mark.parametrize("lengths", [same(1), same(1, 2, 15, 16, 17, 31, 32, 33), same(63, 64, 65, 0, 127, 128, 129), same(300), same(0, 0, 5)])
def test_lengths(H, group, lengths):
    check(H, group, lengths, pad_q=2, pad_k=2, stride_pad=8)


@pytest.mark.parametrize("H,group,n", [(8, 5, 1111), (8, 1, 2100), (1, 16, 2300), (2, 7, 1900), (8, 16, 700)])
def test_long_prompts(H, group, n):
    """A lone prompt, and one of several: its blocks are paired otherwise."""
    check(H, group, same(n))
    check(H, group, same(n, 77, n // 2, 3, n // 3, 900, 800), fused=True)


@pytest.mark.parametrize("H,group", [(1, 33), (1, 129), (2, 255), (1, 256), (1, 300), (2, 1000)])
@pytest.mark.parametrize("lengths", [same(1, 3), same(70), [(5, 200), (1, 1), (33, 40)]])
def test_more_queries_to_a_head_than_a_block_has_rows(H, group, lengths):
    check(H, group, lengths, pad_q=1)
    check(H, group, lengths, window=9, sink=2, join=True)


@pytest.mark.parametrize("lengths", [[(1, 1000)], [(5, 1000), (1, 1), (40, 41)], [(64, 4000)], [(300, 900), (20, 20), (700, 1500)], [(1, 30000)]])
@pytest.mark.parametrize("H,group", [(8, 5), (2, 2)])
def test_chunks_behind_earlier_keys(lengths, H, group):
    check(H, group, lengths, pad_q=1, pad_k=3)


@pytest.mark.parametrize("lengths", [[(5, 3)], [(70, 2), (3, 0), (200, 130)], [(400, 390)] * 17, [(9, 0)]])
def test_more_queries_than_keys(lengths):
    """The first queries see nothing: zeros and -infinity, or the part that is joined."""
    check(8, 5, lengths)
    check(8, 5, lengths, join=True)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (7, 0), (64, 4), (100, 70), (200, 1), (1000, 5), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
@pytest.mark.parametrize("lengths", [same(1, 40, 250), [(70, 900), (3, 77)], WIDE[:13] + [(500, 900)] * 5], ids=["short", "chunks", "wide"])
def test_windows_and_sinks(window, sink, lengths):
    check(8, 5, lengths, window=window, sink=sink)


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.1, 1.0, 3e-39, 0.7])
@pytest.mark.parametrize("lengths", [same(50, 12), WIDE], ids=["short", "wide"])
def test_scales(scale, lengths):
    check(8, 5, lengths, scale=scale)


@pytest.mark.parametrize("lengths", [same(50, 12), WIDE, [(3, 5000)]], ids=["short", "wide", "long"])
@pytest.mark.parametrize("kw", [dict(join=True), dict(f32=True), dict(f32=True, join=True, stride_pad=16), dict(no_lse=True), dict(max_len=1), dict(max_len=100000)],
                         ids=lambda kw: "-".join(kw))
def test_outputs_and_joins(lengths, kw):
    check(8, 5, lengths, **kw)


@pytest.mark.parametrize("lengths", [same(40, 200), [(30, 90)], WIDE], ids=["short", "chunk", "wide"])
@pytest.mark.parametrize("window,sink", [(0, 0), (8, 1)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(lengths, window, sink):
    def poison(k, v):
        at = 0
        for _, m in lengths:
            v[at + m // 3][:, 32:40] = math.inf
            v[at + m // 3][:, 37] = -math.inf
            v[at + m // 2][:, 100] = math.nan
            v[at + m - 1][:, 3] = -math.inf
            at += m
    out, _ = check(8, 5, lengths, window=window, sink=sink, poison=poison)
    assert not torch.isfinite(out[lengths[0][0] - 1]).all()
    if lengths[0][0] == lengths[0][1]:
        assert torch.isfinite(out[0]).all()
    check(8, 5, lengths, window=window, sink=sink, poison=poison, join=True, f32=True)


@pytest.mark.parametrize("lengths", [[(200, 200)], [(30, 90)], [(900, 900)] * 4], ids=["short", "chunk", "wide"])
def test_what_is_not_seen_may_hold_anything(lengths):
    """Keys and values of the last tokens are NaN and infinite: queries before them are what they are without."""
    def poison(k, v):
        at = 0
        for _, m in lengths:
            k[at + m - 2:at + m], v[at + m - 2], v[at + m - 1] = math.nan, math.inf, math.nan
            at += m
    H, group = 8, 5
    out, lse = check(H, group, lengths)
    bad, blse = check(H, group, lengths, poison=poison)
    at = 0
    for n, _ in lengths:
        assert torch.equal(out[at:at + n - 2], bad[at:at + n - 2]) and torch.equal(lse[at:at + n - 2], blse[at:at + n - 2])
        assert torch.isnan(bad[at + n - 1]).all()
        at += n


@pytest.mark.parametrize("lengths", [same(50, 12), WIDE], ids=["short", "wide"])
@pytest.mark.parametrize("kw", [dict(spread=300.0), dict(scale=2.0 ** 20), dict(scale=-2.0 ** 40), dict(size=1e33), dict(size=1e-30)], ids=str)
def test_scores_and_values_of_other_sizes(lengths, kw):
    check(8, 5, lengths, **kw)


@pytest.mark.parametrize("seed", range(8))
def test_random_batches(seed):
    rng = np.random.default_rng(seed)
    H, group = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 4, 5, 7, 8, 16]))
    lengths = []
    for _ in range(int(rng.integers(1, 14))):
        n = int(rng.choice([0, 1, 2, int(rng.integers(1, 700))]))
        lengths.append((n, max(0, n + int(rng.choice([0, 0, -1, int(rng.integers(0, 500))])))))
    kw = dict(window=int(rng.integers(1, 400)), sink=int(rng.integers(0, 90))) if rng.random() < 0.5 else {}
    check(H, group, lengths, seed=seed, pad_q=int(rng.integers(0, 4)), pad_k=int(rng.integers(0, 4)), stride_pad=8 * int(rng.integers(0, 3)), join=bool(rng.random() < 0.4), **kw)


@pytest.mark.parametrize("n_seqs", [62, 63, 64, 65, 127, 128, 129, 300])
def test_many_sequences(n_seqs):
    """As many starts as lanes and more, with sequences that have nothing among them."""
    lengths = [(0, 3) if s % 7 == 2 else (0, 0) if s % 7 == 4 else (1 + 37 * s % 90, 1 + 37 * s % 90 + (s % 3) * 11) for s in range(n_seqs)]
    check(2, 5, lengths, pad_q=1, pad_k=1)


def test_rows_as_far_apart_as_they_may_be():
    """Strides of 2^24 elements: a whole step of 64 tokens, and one that ends before."""
    H, Hq, n, stride = 2, 6, 100, 1 << 24
    g = torch.Generator().manual_seed(3)
    q, k, v = (bf(torch.randn(n, h * 128, generator=g)) for h in (Hq, H, H))
    big = torch.zeros(n * stride - stride + 2 * H * 128, dtype=torch.bfloat16, device="cuda")
    rows = [big[i * H * 128:].as_strided((n, H * 128), (stride, 1)) for i in (0, 1)]
    for d, x in zip(rows, (k, v)):
        d.copy_(x.cuda())
    dq, s = q.cuda(), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(n, Hq * 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, Hq, device="cuda")
    kv, batch = tdk.tdk_kv_create(tdk.model(1, H)), tdk.prompt_batch(1, n, n, n, s, s)
    space = torch.empty(max(256, tdk.tdk_prompt_attend_workspace_bytes(kv, batch, Hq)), dtype=torch.uint8, device="cuda")
    tdk.tdk_prompt_attend(kv, batch, tdk.prompt_attend_io(dq, Hq * 128, Hq, rows[0], stride, rows[1], stride, 0.09, out, Hq * 128, lse, space, space.numel()), stream())
    torch.cuda.synchronize()
    want, wlse, mass, scores = ph.attend([(n, n)], q.double().reshape(n, Hq, 128), k.double().reshape(n, H, 128), v.double().reshape(n, H, 128), 0.09)
    tol, ltol = kh.tolerance(want, wlse, mass, scores, n)
    assert far(out.cpu().double().reshape(n, Hq, 128), want, tol) == 0 and far(lse.cpu().double(), wlse, ltol) == 0


def test_results_repeat_bit_for_bit():
    for lengths in (same(50, 12), WIDE, [(3, 5000)]):
        first = check(8, 5, lengths)
        again = check(8, 5, lengths)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_starts_are_cut_to_the_rows_there_are():
    """Starts beyond the buffers and below zero: no row outside is touched."""
    H, Hq, N, M = 2, 4, 20, 30
    g = torch.Generator().manual_seed(1)
    q, k, v = (bf(torch.randn(n, h * 128, generator=g)).cuda() for n, h in ((N, Hq), (M, H), (M, H)))
    out = torch.full((N + 8, Hq * 128), 9.0, dtype=torch.bfloat16, device="cuda")
    qs = torch.tensor([-5, 7, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ks = torch.tensor([-2 ** 31, 11, 2 ** 30], dtype=torch.int32, device="cuda")
    kv, batch = tdk.tdk_kv_create(tdk.model(1, H)), tdk.prompt_batch(2, N, M, 30, qs, ks)
    space = torch.empty(max(256, tdk.tdk_prompt_attend_workspace_bytes(kv, batch, Hq)), dtype=torch.uint8, device="cuda")
    tdk.tdk_prompt_attend(kv, batch, tdk.prompt_attend_io(q, Hq * 128, Hq, k, H * 128, v, H * 128, 0.1, out, Hq * 128, None, space, space.numel()), stream())
    torch.cuda.synchronize()
    want, wlse, mass, big = ph.attend([(7, 11), (13, 19)], q.cpu().double().reshape(N, Hq, 128), k.cpu().double().reshape(M, H, 128), v.cpu().double().reshape(M, H, 128), 0.1)
    tol, _ = kh.tolerance(want, wlse, mass, big, 30)
    assert ((out[:N].cpu().double().reshape(N, Hq, 128) - want).abs() <= tol).all() and (out[N:] == 9.0).all()
