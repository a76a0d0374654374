"""Rounds made with scaled frequencies, through every call that turns rows: re-rotation, encode, decode, layerwise restore, restore at new offsets, and attention's
turned queries; both layouts of the pairs, identity layouts and segments.

All frequencies divided by 8 at eight times the distances are the same angles, bit for bit (8 is a power of two).  So each round has a twin: the same pages, every agent
(every segment) eight times as far from its master, on a handle whose frequencies are divided by 8.  The oracle runs the plain round, the library the
twin; results are equal bit for bit, attention within attend_bounds."""
import copy

import numpy as np
import pytest

import attend_bounds as ab
from paper_2604_03143_amd import workload as wl
from helpers import OracleRun

pytestmark = pytest.mark.gpu
F, POS0 = 8, 5
FORMS = pytest.mark.parametrize("style,T,segments", [(0, 16, False), (1, 16, False), (0, 32, False), (1, 32, True), (0, 16, True), (1, 16, True)])


def make(T, segments, layers=1, stream=121, H=8, grow=0):
    """A round whose distances are multiples of the page size, so that its twin has the same rows in the same places of its pages."""
    spec = wl.RoundSpec("turned", stream, layers, H, 128, T, 1.0e6, 2, 3, 5, 2 * T if segments else 2 * T + 7, 0, 0, 0.25)
    hist = np.array([0, 3, 40, 1, 7, 13], np.int64) * T + (320 if segments else POS0) + grow
    rnd = wl.make_round(spec, hist=hist)
    if segments:
        wl.permute_blocks(rnd)
    else:
        rnd.master_pos0 = np.full(rnd.n_sessions, POS0, np.int64)
    return spec, rnd


def far(rnd, agent, pos, src=0):
    """Eight times as far from where the master has that token."""
    at = int(rnd.master_pos0[rnd.agent_session[agent]]) + np.asarray(src, np.int64)
    return at + F * (np.asarray(pos, np.int64) - at)


def twin(rnd):
    T, new = rnd.spec.page_tokens, copy.copy(rnd)
    new.agent_pos0 = np.array([far(rnd, i, p) for i, p in enumerate(rnd.agent_pos0)], np.int64)
    new.block_tables, new.segments = [], None if rnd.segments is None else []
    for i, old in enumerate(rnd.block_tables):
        S = int(rnd.span_tokens[rnd.agent_session[i]])
        runs = np.array([[0, rnd.agent_pos0[i], S]], np.int64) if rnd.segments is None else rnd.segments[i]
        moved = np.stack([runs[:, 0], far(rnd, i, runs[:, 1], runs[:, 0]), runs[:, 2]], 1)
        assert ((moved[:, 1] - runs[:, 1]) % T == 0).all() and (moved[:, 1] >= 0).all()
        table = np.full(int((moved[:, 1] + moved[:, 2]).max() + T - 1) // T, rnd.dummy_page, np.int32)
        for (_, a, n), (_, b, _) in zip(runs, moved):
            for lp in range(a // T, (a + n - 1) // T + 1):
                table[lp + (b - a) // T] = old[lp]
        new.block_tables.append(table)
        if rnd.segments is not None:
            new.segments.append(moved)
    return new


def create(rnd, style, diff_pos0=None, segment_diff_pos=None):
    from paper_2604_03143_amd import tdk
    sp = rnd.spec
    # (the magnitude is the appended keys' own: a round does not apply it again)
    rope = tdk.rope(128, tdk.ROPE_SCALE_LINEAR, float(F), magnitude=1.3)
    mdl = tdk.model(sp.num_layers, sp.num_kv_heads, sp.head_dim, sp.page_tokens, sp.rope_theta, style)
    return tdk.tdk_round_create_rope(mdl, rope, rnd.span_tokens, rnd.master_pos0, rnd.agent_session, rnd.agent_pos0, rnd.block_tables, diff_pos0, rnd.segments, segment_diff_pos)


def gpu_run(rnd, o, style, **kw):
    """The twin on the GPU, with the plain round's masters."""
    import gpu_helpers as gh
    g = gh.GpuRun(rnd, style=style, mk=o.mk, mv=o.mv, layer=o.layer)
    g.r.destroy()
    g.rnd, g.r = twin(rnd), create(twin(rnd), style, **kw)
    return g


@FORMS
def test_rerotate_encode_and_decode(tdo, style, T, segments):
    import gpu_helpers as gh
    spec, rnd = make(T, segments)
    o = OracleRun(tdo, rnd, style=style)
    g = gpu_run(rnd, o, style)
    try:
        o.rerotate()
        g.rerotate()
        gk, gv = g.pool()
        assert np.array_equal(gk, o.pk) and np.array_equal(gv, o.pv)
        assert not np.array_equal(o.pk, wl.pool_host(rnd, 0)[0])
        o.perturb()
        g.set_pool(o.pk, o.pv)
        od, gd = o.encode(), g.encode()
        gh.assert_diff_equal(gd, od, rnd.n_agents)
        listed, pages = int(od.offset[-1]), sum(-(-int(rnd.span_tokens[s]) // T) for s in rnd.agent_session)
        assert 0 < listed < pages                      # (other angles than the oracle's would list every page but those of agents that have not moved)
        g.set_pool(*wl.pool_host(rnd, 0))
        g.decode(gd)
        opk, opv = wl.pool_host(rnd, 0)
        o.decode(od, opk, opv)
        gk, gv = g.pool()
        assert np.array_equal(gk, opk) and np.array_equal(gv, opv)
        mask = wl.shared_row_mask(rnd)
        assert np.array_equal(gk[mask], o.pk[mask]) and np.array_equal(gv[mask], o.pv[mask])
    finally:
        g.close()


@FORMS
def test_layerwise_restore(tdo, style, T, segments):
    import torch
    import gpu_helpers as gh
    from paper_2604_03143_amd import tdk
    L = 3
    spec, rnd = make(T, segments, layers=L, stream=122)
    runs = [OracleRun(tdo, rnd, layer=i, style=style) for i in range(L)]
    diffs = []
    for o in runs:
        o.rerotate(); o.perturb()
        diffs.append(o.encode())
    hk, hv = ([torch.from_numpy(x.view(np.int16)).pin_memory() for x in xs] for xs in ([o.mk for o in runs], [o.mv for o in runs]))
    size = hk[0].numel() * 2
    stage = [torch.zeros(size // 2, dtype=torch.int16, device="cuda") for _ in range(4)]
    pools = [[gh.up(x) for x in wl.pool_host(rnd, i)] for i in range(L)]
    keep, dd = [], []
    for d in diffs:
        n = int(d.offset[-1])
        t = [torch.from_numpy(d.count).cuda(), torch.from_numpy(d.offset).cuda(), torch.from_numpy(d.idx[:n].copy()).cuda(), gh.up(d.payload[:n].copy()),
             torch.zeros(1, dtype=torch.int32, device="cuda")]
        keep.append(t)
        dd.append(tdk.diff(t[0], t[1], t[2], t[3], n, t[4]))
    r, comp, cp = create(twin(rnd), style), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    try:
        tdk.tdk_restore_layers(r, 0, hk, hv, [tdk.layer_io(None, None, k, v, rnd.pool_pages) for k, v in pools], dd, tdk.pingpong(*stage, size), comp.cuda_stream, cp.cuda_stream)
        comp.synchronize(); cp.synchronize()
        for i, o in enumerate(runs):
            pk, pv = wl.pool_host(rnd, i)
            o.decode(diffs[i], pk, pv)
            assert np.array_equal(gh.down16(pools[i][0]), pk) and np.array_equal(gh.down16(pools[i][1]), pv), i
    finally:
        torch.cuda.synchronize()
        r.destroy()


def moved(rnd, T):
    """Where each agent's rows (segments) were when the mirrors were stored: some pages elsewhere, one agent where it is."""
    by = [0, 1, 2, 5, 3, 1]
    if rnd.segments is None:
        return dict(diff_pos0=np.maximum(rnd.agent_pos0 - np.array(by, np.int64) * T, POS0))
    return dict(diff_pos0=rnd.agent_pos0, segment_diff_pos=[x[:, 1] - T * ((by[i] + np.arange(len(x))) % 4) for i, x in enumerate(rnd.segments)])


def moved_twin(rnd, was):
    """The same eight times as far from where the rows are now."""
    new = twin(rnd)
    if rnd.segments is None:
        return dict(diff_pos0=new.agent_pos0 - F * (rnd.agent_pos0 - was["diff_pos0"]))
    return dict(diff_pos0=new.agent_pos0, segment_diff_pos=[y[:, 1] - F * (x[:, 1] - p) for x, y, p in zip(rnd.segments, new.segments, was["segment_diff_pos"])])


def stored(tdo, rnd, style):
    """Mirrors as the oracle stores them."""
    import torch
    import gpu_helpers as gh
    from paper_2604_03143_amd import tdk
    o = OracleRun(tdo, rnd, style=style)
    o.rerotate(); o.perturb()
    d = o.encode()
    n = int(d.offset[-1])
    t = [torch.from_numpy(d.count).cuda(), torch.from_numpy(d.offset).cuda(), torch.from_numpy(d.idx[:n].copy()).cuda(), gh.up(d.payload[:n].copy()),
         torch.zeros(1, dtype=torch.int32, device="cuda")]
    return o, d, t, tdk.diff(t[0], t[1], t[2], t[3], n, t[4])


@FORMS
def test_restore_at_new_offsets(tdo, style, T, segments):
    from paper_2604_03143_amd import tdk
    spec, rnd = make(T, segments, stream=123)
    was = moved(rnd, T)
    o, d, keep, dd = stored(tdo, rnd, style)
    opk, opv = wl.pool_host(rnd, 0)
    tdo.diff_decode(o.g, tdo.HostRound(rnd, **was), o.mk, o.mv, opk, opv, d)
    g = gpu_run(rnd, o, style, **moved_twin(rnd, was))
    try:
        tdk.tdk_diff_decode(g.r, 0, g.io, dd, g.stream)
        gk, gv = g.pool()
        assert np.array_equal(gk, opk) and np.array_equal(gv, opv)
        assert not np.array_equal(opk, o.pk)           # (the payload's rows did turn)
    finally:
        g.close()


@FORMS
@pytest.mark.parametrize("n_q,Hq", [(1, 40), (5, 16)])
def test_attention_with_turned_queries(tdo, style, T, segments, n_q, Hq):
    import torch
    import gpu_helpers as gh
    from paper_2604_03143_amd import tdk
    spec, rnd = make(T, segments, stream=124)
    was = moved(rnd, T)
    o, d, keep, dd = stored(tdo, rnd, style)
    q = wl.f32_to_bf16_bits(np.random.default_rng(n_q).standard_normal((rnd.n_agents, n_q, Hq, 128)).astype(np.float32))
    scale = 0.5                                        # (sharp weights: rows that are turned otherwise move far outside the bound)
    bounds = ab.expected_and_bounds(tdo, o.g, tdo.HostRound(rnd, **was), o.mk, o.mv, d, q, n_q, Hq, scale)
    g = gpu_run(rnd, o, style, **moved_twin(rnd, was))
    try:
        need = tdk.tdk_attend_workspace_bytes(g.r, n_q, Hq)
        space = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        out = torch.full((rnd.n_agents, n_q, Hq, 128), float("nan"), device="cuda")
        lse = torch.full((rnd.n_agents, n_q, Hq), float("nan"), device="cuda")
        dq = gh.up(q)
        tdk.tdk_attend_shared(g.r, 0, g.io, dd, tdk.attend_io(dq, n_q, Hq, scale, out, lse, space, need), g.stream)
        torch.cuda.synchronize()
        got = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        ab.assert_within(*got, *bounds, what=(style, T, segments, n_q, Hq))
        # the plain round's positions with plain frequencies are another thing than the twin's positions with them
        if n_q == 1:
            wrong = ab.expected_and_bounds(tdo, o.g, tdo.HostRound(twin(rnd), **moved_twin(rnd, was)), o.mk, o.mv, d, q, n_q, Hq, scale)
            assert not ab.within(*got, *wrong)
    finally:
        g.close()


@pytest.mark.parametrize("interleaved", [False, True])
def test_plain_positions_are_plain_rounds(interleaved):
    """tdk_rope that changes nothing: the rows of tdk_round_create, bit for bit."""
    import torch
    import gpu_helpers as gh
    from paper_2604_03143_amd import tdk
    spec, rnd = make(16, False, stream=125)
    a, b = gh.GpuRun(rnd, style=int(interleaved)), gh.GpuRun(rnd, style=int(interleaved))
    b.r.destroy()
    mdl = tdk.model(spec.num_layers, spec.num_kv_heads, 128, 16, spec.rope_theta, int(interleaved))
    b.r = tdk.tdk_round_create_rope(mdl, tdk.rope(), rnd.span_tokens, rnd.master_pos0, rnd.agent_session, rnd.agent_pos0, rnd.block_tables)
    try:
        a.rerotate(); b.rerotate()
        torch.cuda.synchronize()
        assert torch.equal(a.pk, b.pk) and torch.equal(a.pv, b.pv)
    finally:
        a.close(); b.close()


@pytest.mark.parametrize("scaling", ["turns", "index"])
def test_interleaved_rows_turn_by_the_same_frequencies(scaling):
    """The two scalings that differ from pair to pair, pairs side by side: each agent's rows by the distance times its pair's frequency."""
    import torch
    import gpu_helpers as gh
    import rope_helpers as rh
    from paper_2604_03143_amd import tdk
    from test_gpu_rope import INDEX, SCALINGS, TURNS
    s = TURNS if scaling == "turns" else INDEX
    spec, rnd = make(16, False, stream=126, H=3, grow=9000)
    g = gh.GpuRun(rnd, style=tdk.ROPE_INTERLEAVED)
    g.r.destroy()
    rope = tdk.rope(128, SCALINGS[scaling], s["factor"], s["original"], s["low"], s["high"])
    g.r = tdk.tdk_round_create_rope(tdk.model(1, 3, 128, 16, 1.0e6, tdk.ROPE_INTERLEAVED), rope, rnd.span_tokens, rnd.master_pos0, rnd.agent_session, rnd.agent_pos0, rnd.block_tables)
    f = rh.frequencies(1.0e6, 128, **s)
    try:
        g.rerotate()
        gk, _ = g.pool()
        mk = g.mk.cpu().view(torch.bfloat16).float().numpy()
        for i in range(rnd.n_agents):
            ses = int(rnd.agent_session[i])
            rows = mk[int(rnd.master_row0[ses]):int(rnd.master_row0[ses + 1])].reshape(-1, 3, 128)
            want = torch.as_tensor(rh.rotate(rows, np.full(len(rows), int(rnd.agent_pos0[i]) - POS0), f, 128, True)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
            assert np.array_equal(gk.reshape(-1, 3, 128)[rnd.dst_rows(i)], want), i
    finally:
        g.close()
