"""tdk_kv_* as programs use them: together with the rounds' calls, captured in graphs, on several streams, step after step."""
import math

import numpy as np
import pytest
import torch

import gpu_helpers as gh
import kv_helpers as kh
from paper_2604_03143_amd import tdk, workload as wl

pytestmark = pytest.mark.gpu
D, H, HQ, SCALE = 128, 8, 40, 1 / math.sqrt(128)


def bf(x):
    return torch.as_tensor(x).to(torch.bfloat16)


def cur():
    return torch.cuda.current_stream().cuda_stream


class Step:
    """One batch over a pool of pages: new rows, their append and their attention, with buffers of its own."""

    def __init__(self, fmt, b, seed, window=0, sink=0, heads=H, q_heads=HQ):
        g = torch.Generator().manual_seed(seed)
        self.b, self.fmt, self.window, self.sink, self.hq = b, fmt, window, sink, q_heads
        self.kv = tdk.tdk_kv_create(tdk.model(1, heads, D, b.T), fmt)
        if fmt == tdk.KV_BF16:
            self.pools = [bf(torch.randn(b.pool_pages, b.T, heads, D, generator=g)).cuda() for _ in range(2)]
        else:
            self.pools = [kh.pack4(*kh.to4(torch.randn(b.pool_pages, b.T, heads, D, generator=g)), b.T).cuda() for _ in range(2)]
        self.q, self.k, self.v = (bf(torch.randn(b.n, h * D, generator=g)).cuda() for h in (q_heads, heads, heads))
        self.q_rot = torch.zeros_like(self.q)
        self.out = torch.zeros(b.n, q_heads * D, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.zeros(b.n, q_heads, device="cuda")
        self.cache = tdk.kv_cache(*self.pools, b.pool_pages)
        self.batch = b.struct(tdk)
        self.arrays = b.d                  # (the batch holds addresses only)
        self.need = tdk.tdk_kv_attend_workspace_bytes(self.kv, self.batch, q_heads)
        self.space = torch.empty(self.need + 256, dtype=torch.uint8, device="cuda")
        self.rows = tdk.kv_rows(self.k, self.v, heads * D, heads * D, q=self.q, q_stride=q_heads * D, n_q_heads=q_heads, q_out=self.q_rot, q_out_stride=q_heads * D)
        self.io = tdk.kv_attend_io(self.q_rot, q_heads * D, q_heads, SCALE, self.out, q_heads * D, self.lse, self.space, self.need, window, sink)

    def run(self, stream=None):
        s = cur() if stream is None else stream
        tdk.tdk_kv_append(self.kv, self.cache, self.batch, self.rows, s)
        tdk.tdk_kv_attend(self.kv, self.cache, self.batch, self.io, s)

    def result(self):
        torch.cuda.synchronize()
        return [t.cpu().clone() for t in (self.out, self.lse, self.q_rot, *self.pools)]


def same(x, y):
    return all(torch.equal(a.view(torch.uint8) if a.dtype == torch.uint8 else a.view(torch.int16 if a.element_size() == 2 else torch.int32),
                           b.view(torch.uint8) if b.dtype == torch.uint8 else b.view(torch.int16 if b.element_size() == 2 else torch.int32)) for a, b in zip(x, y))


SHAPES = [[(40, 1), (0, 1), (333, 1)], [(5, 9), (70, 3)], [(0, 60), (100, 40)], [(4000, 1)], [(3000, 70)]]


@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4], ids=["bf16", "mxfp4"])
@pytest.mark.parametrize("lengths", SHAPES)
def test_graphs_replay_with_new_lengths_and_rows(fmt, lengths):
    """A captured step, replayed with other rows, other (shorter) lengths and eager work in between: every replay as the eager call."""
    b = kh.Batch(lengths, 16, 3)
    s, e = Step(fmt, b, 5), Step(fmt, b, 5)
    s.run()
    torch.cuda.synchronize()
    for p, o in zip(s.pools, e.pools):
        p.copy_(o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for r in range(4):
        g = torch.Generator().manual_seed(100 + r)
        for t, u in zip((s.q, s.k, s.v), (e.q, e.k, e.v)):
            x = bf(torch.randn(t.shape, generator=g)).cuda()
            t.copy_(x)
            u.copy_(x)
        lens = torch.tensor([max(n, h + n - 3 * r) for h, n in lengths], dtype=torch.int32).cuda()
        s.space.fill_(0xFF)
        for x in (s, e):
            x.out.zero_()
            x.arrays[1].copy_(lens)
        torch.cuda.synchronize()
        graph.replay()
        got = s.result()
        e.run()
        assert same(got, e.result()), r


@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4], ids=["bf16", "mxfp4"])
def test_two_streams_and_two_graphs_at_once(fmt):
    """Steps that share a handle, with workspaces of their own, on two streams and as two graphs: each as if alone."""
    pairs = [Step(fmt, kh.Batch([(3000, 1), (17, 1)], 16, 1), 2), Step(fmt, kh.Batch([(900, 5), (2100, 2)], 16, 7), 8)]
    for p in pairs[1:]:
        p.kv = pairs[0].kv
    start = [[t.clone() for t in p.pools] for p in pairs]
    want = []
    for p in pairs:
        p.run()
        want.append(p.result())
    streams = [torch.cuda.Stream() for _ in pairs]
    graphs = []
    for p, st in zip(pairs, streams):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            p.run()
        graphs.append(gr)
    for way in range(2):
        for p, old in zip(pairs, start):
            for t, u in zip(p.pools, old):
                t.copy_(u)
            p.out.zero_()
            p.space.fill_(0xFF)
        torch.cuda.synchronize()
        for _ in range(3):
            for p, st, gr in zip(pairs, streams, graphs):
                with torch.cuda.stream(st):
                    p.run() if way == 0 else gr.replay()
        for p, w in zip(pairs, want):
            assert same(p.result(), w)


def test_results_repeat_bit_for_bit():
    for lengths in SHAPES:
        s = Step(tdk.KV_BF16, kh.Batch(lengths, 32, 3), 5, window=100, sink=2)
        s.run()
        first = s.result()
        for _ in range(3):
            s.space.fill_(0x7F)
            s.run()
            assert same(first, s.result())


def test_one_sequence_twice_and_pages_in_common():
    """Two sequences of a batch may read the same pages (a shared prefix): each as if alone."""
    b = kh.Batch([(100, 1), (100, 1)], 16, 5)
    b.table[1, :6] = b.table[0, :6]                    # 96 tokens in common
    s = Step(tdk.KV_BF16, b, 6)
    s.run()
    out, lse, *_ = s.result()
    k, v = (p.cpu().double() for p in s.pools)
    want, wlse, mass, big = kh.attend(b, k, v, s.q_rot.cpu().double().reshape(2, HQ, D), SCALE)
    tol, ltol = kh.tolerance(want, wlse, mass, big, 101)
    assert ((out.double().reshape(2, HQ, D) - want).abs() <= tol).all() and ((lse.double() - wlse).abs() <= ltol).all()


def test_offsets_beyond_32_bits():
    """A pool of over 4 GiB a plane, its last pages in use."""
    T, heads = 16, 8
    pages = (5 << 30) // (T * heads * 256)
    pk, pv = (torch.zeros(pages, T, heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    b = kh.Batch([(20, 2), (3, 1)], T, 5)
    b.table = np.where(b.table >= 0, pages - 1 - b.table, b.table).astype(np.int32)
    b.pool_pages = pages
    g = torch.Generator().manual_seed(4)
    used = sorted({int(p) for p in b.table[b.table >= 0]})
    for p in used:
        pk[p] = bf(torch.randn(T, heads, D, generator=g)).cuda()
        pv[p] = bf(torch.randn(T, heads, D, generator=g)).cuda()
    kv = tdk.tdk_kv_create(tdk.model(1, heads, D, T))
    cache, batch = tdk.kv_cache(pk, pv, pages), b.struct(tdk)
    q, k, v = (bf(torch.randn(b.n, heads * D, generator=g)).cuda() for _ in range(3))
    tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(k, v, heads * D, heads * D, q=q, q_stride=heads * D, n_q_heads=heads, q_out=q, q_out_stride=heads * D), cur())
    out, lse = torch.zeros_like(q), torch.zeros(b.n, heads, device="cuda")
    space = torch.empty(max(256, tdk.tdk_kv_attend_workspace_bytes(kv, batch, heads)), dtype=torch.uint8, device="cuda")
    tdk.tdk_kv_attend(kv, cache, batch, tdk.kv_attend_io(q, heads * D, heads, SCALE, out, heads * D, lse, space, space.numel()), cur())
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    tdk.tdk_kv_read(kv, cache, batch, tdk.kv_rows(k2, v2, heads * D, heads * D), cur())
    torch.cuda.synchronize()
    assert torch.equal(v2, v)
    small = {p: i for i, p in enumerate(used)}
    c = kh.Batch(b.lengths, T, 5)
    c.table = np.array([[small.get(int(p), -1) for p in row] for row in b.table], np.int32)
    kk, vv = (torch.stack([x[p] for p in used]).cpu().double() for x in (pk, pv))
    c.pool_pages = len(used)
    want, wlse, mass, big = kh.attend(c, kk, vv, q.cpu().double().reshape(b.n, heads, D), SCALE)
    tol, ltol = kh.tolerance(want, wlse, mass, big, 22)
    assert ((out.cpu().double().reshape(b.n, heads, D) - want).abs() <= tol).all() and ((lse.cpu().double() - wlse).abs() <= ltol).all()




@pytest.mark.parametrize("fmt", [tdk.KV_BF16, tdk.KV_MXFP4], ids=["bf16", "mxfp4"])
def test_a_round_and_the_agents_own_tokens(fmt):
    """What a layer does in a round: the shared span is attended to from master + diff, private histories and new tokens in the agents'
    own pages, joined; the new tokens are appended first; then one token more; and the finished output becomes a master again.

    bf16: the private pages are the round's own pool, where the span is restored too, so one call over everything says the same.  4 bits: the
    private pages are a cache of their own, in which the span has no pages at all."""
    spec = wl.RoundSpec("kvuse", 61, 1, H, D, 16, 1.0e6, 1, 4, 3, 50, 5, 120, 0.2)
    rnd = wl.make_round(spec)
    S, T, A = 150, 16, rnd.n_agents
    hist = [int(p) for p in rnd.agent_pos0]
    n_new = 6
    g = torch.Generator().manual_seed(9)
    # the round's pool: pages of its own for histories too, and for the tokens behind the span
    pages = [-(-(h + S + n_new + 2) // T) for h in hist]
    order = np.random.default_rng(3).permutation(sum(pages) + 2)
    tables, at = [], 0
    for p in pages:
        tables.append(order[at:at + p].astype(np.int32))
        at += p
    pool_pages = sum(pages) + 2
    pk, pv = (bf(torch.randn(pool_pages, T, H, D, generator=g)).cuda() for _ in range(2))
    mk, mv = (bf(torch.randn(S, H, D, generator=g)).cuda() for _ in range(2))
    r = tdk.tdk_round_create(tdk.model(1), [S], [0], [0] * A, hist, tables)
    io = tdk.layer_io(mk, mv, pk, pv, pool_pages)
    tdk.tdk_rerotate_round(r, 0, io, cur())
    torch.cuda.synchronize()
    for a in range(A):                                 # refreshed pages
        for j in range(32 * a, 32 * a + 20):
            p = hist[a] + j
            pk[int(tables[a][p // T]), p % T] += bf(0.5 * torch.randn(H, D, generator=g)).cuda()
    d = gh.DevDiff(A, A * 10, 2 * T * H * D)
    tdk.tdk_diff_encode(r, 0, io, 1e-2, d.c, cur())

    b = kh.Batch([(h + S, n_new) for h in hist], T, 1)
    b.stride = max(pages)
    b.table = np.full((A, b.stride), -1, np.int32)
    for a in range(A):
        b.table[a, :pages[a]] = tables[a]
    b.pool_pages = pool_pages
    kv = tdk.tdk_kv_create(tdk.model(1), fmt)
    if fmt == tdk.KV_BF16:
        own_k, own_v = pk, pv
    else:
        own_k, own_v = (kh.pack4(*kh.to4(x.float().cpu()), T).cuda() for x in (pk, pv))
        for a in range(A):                             # pages that hold nothing but the shared span are not there
            b.table[a, -(-hist[a] // T):(hist[a] + S) // T] = -1
    hole = torch.tensor([[h, h + S] for h in hist], dtype=torch.int32).cuda()
    q, k, v = (bf(torch.randn(b.n, h * D, generator=g)).cuda() for h in (HQ, H, H))
    cache = tdk.kv_cache(own_k, own_v, pool_pages)

    def step(b, q, k, v):
        n_q = b.n // A
        batch = b.struct(tdk)
        tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(k, v, H * D, H * D, q=q, q_stride=HQ * D, n_q_heads=HQ, q_out=q, q_out_stride=HQ * D), cur())
        part_out, part_lse = torch.empty(b.n, HQ, D, device="cuda"), torch.empty(b.n, HQ, device="cuda")
        w = torch.empty(tdk.tdk_attend_workspace_bytes(r, n_q, HQ), dtype=torch.uint8, device="cuda")
        tdk.tdk_attend_shared(r, 0, io, d.c, tdk.attend_io(q, n_q, HQ, SCALE, part_out, part_lse, w, w.numel()), cur())
        out, lse = torch.empty(b.n, HQ * D, dtype=torch.bfloat16, device="cuda"), torch.empty(b.n, HQ, device="cuda")
        need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, HQ)
        space = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        tdk.tdk_kv_attend(kv, cache, batch, tdk.kv_attend_io(q, HQ * D, HQ, SCALE, out, HQ * D, lse, space, need, hole=hole, part_out=part_out,
                                                             part_lse=part_lse), cur())
        torch.cuda.synchronize()
        # everything at once, in 64 bits: the span's tokens from the round's pool (the mirrors as they are), the others from the cache
        kk, vv = (x.cpu() for x in (pk, pv))
        if fmt == tdk.KV_MXFP4:
            f = [kh.from4(*kh.unpack4(x.cpu(), T)) for x in (own_k, own_v)]
            kk, vv = kk.double(), vv.double()
            for a in range(A):
                for p in list(range(hist[a])) + list(range(hist[a] + S, int(b.lens[a]))):
                    pg = int(tables[a][p // T])
                    kk[pg, p % T], vv[pg, p % T] = f[0][pg, p % T], f[1][pg, p % T]
        full = kh.Batch(b.lengths, T, 1)
        full.table, full.stride, full.pool_pages = np.full((A, max(pages)), -1, np.int32), max(pages), pool_pages
        for a in range(A):
            full.table[a, :pages[a]] = tables[a]
        want, wlse, mass, big = kh.attend(full, kk.double(), vv.double(), q.cpu().double().reshape(b.n, HQ, D), SCALE)
        # the span's part comes from queries that are turned back and rounded to bf16 (2^-8 of a score's terms) and from weights rounded to
        # bf16, a hundredth of the largest |V| by the header; the join adds nothing that counts
        worst = float(vv.double().abs().max())
        assert float((out.cpu().double().reshape(b.n, HQ, D) - want).abs().max()) <= 1e-2 * worst + 2.0 ** -8 * float(want.abs().max())
        assert float((lse.cpu().double() - wlse).abs().max()) <= 2.0 ** -8 * big + 1e-3
        return out

    step(b, q, k, v)
    one = kh.Batch([(h + S + n_new, 1) for h in hist], T, 1)
    one.table, one.stride, one.pool_pages = b.table, b.stride, b.pool_pages
    q1, k1, v1 = (bf(torch.randn(A, h * D, generator=g)).cuda() for h in (HQ, H, H))
    step(one, q1, k1, v1)
    # agent 0's new tokens leave the cache as the next round's master
    outk, outv = (torch.empty(n_new + 1, H * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    last = kh.Batch([(hist[0] + S, n_new + 1)], T, 1)
    last.table, last.stride, last.pool_pages = b.table[:1], b.stride, pool_pages
    tdk.tdk_kv_read(kv, cache, last.struct(tdk), tdk.kv_rows(outk, outv, H * D, H * D), cur())
    torch.cuda.synchronize()
    src_k, src_v = torch.cat((k[:n_new], k1[:1])).float().cpu().numpy().reshape(-1, H, D), torch.cat((v[:n_new], v1[:1])).cpu().reshape(-1, H, D)
    pos = [hist[0] + S + t for t in range(n_new + 1)]
    rk = torch.from_numpy(kh.rotate(src_k, pos, 1e6, False))
    if fmt == tdk.KV_BF16:
        assert torch.equal(outk.cpu().reshape(-1, H, D), bf(rk)) and torch.equal(outv.cpu().reshape(-1, H, D), src_v)
    else:
        assert torch.equal(outk.cpu().reshape(-1, H, D).double(), kh.from4(*kh.to4(rk))) and torch.equal(outv.cpu().reshape(-1, H, D).double(), kh.from4(*kh.to4(src_v.float())))
    # and serve one: re-rotated to other agents' offsets
    r2 = tdk.tdk_round_create(tdk.model(1), [n_new + 1], [pos[0]], [0], [7], [np.array([0, 1], np.int32)])
    p2 = [torch.zeros(2, T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tdk.tdk_rerotate_round(r2, 0, tdk.layer_io(outk, outv, *p2, 2), cur())
    torch.cuda.synchronize()
    assert torch.equal(p2[1].reshape(-1, H * D)[7:7 + n_new + 1].cpu(), outv.cpu())
    r2.destroy()
    r.destroy()
