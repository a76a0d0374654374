"""tdk_kv_*: batches of unusual shapes, and calls at the same time from several host threads."""
import threading

import numpy as np
import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk
from test_gpu_kv import FORMATS, bf, bits, check_append, check_attend, handle, pools, stream

pytestmark = pytest.mark.gpu


@FORMATS
@pytest.mark.parametrize("lengths", [[(100, 1)] * 40 + [(50, 300)], [(50, 90)] + [(70, 1)] * 7, [(10, 200), (0, 1), (300, 1), (0, 0), (5, 130)]])
def test_prompts_and_single_tokens_in_one_batch(fmt, lengths):
    check_attend(fmt, 2, 5, 16, lengths)


@FORMATS
@pytest.mark.parametrize("lengths", [[(-3, 5), (4, 1)], [(-40, 60), (-1, 1), (30, 2)], [(-200, 230)], [(-5, 3), (2, 2)]])
@pytest.mark.parametrize("join", [False, True])
def test_more_new_tokens_than_the_sequence_is_long(fmt, lengths, join):
    """Tokens in front of position 0 see nothing."""
    check_attend(fmt, 2, 3, 16, lengths, join=join, pad=1)


@FORMATS
def test_more_sequences_than_two_rounds_of_the_search_probe(fmt):
    rng = np.random.default_rng(8)
    lengths = [(int(h), int(n)) for h, n in zip(rng.integers(0, 20, 4500), rng.integers(0, 2, 4500))]
    check_append(fmt, 1, 2, 16, False, 1e6, lengths)
    check_attend(fmt, 1, 2, 16, lengths)


@FORMATS
@pytest.mark.parametrize("lengths", [[(40, 1), (0, 2)], [(10, 90), (3, 1)], [(3000, 1)]])
def test_rows_in_front_of_the_first_sequence_stay_as_they_are(fmt, lengths):
    """q_start[0] = 3: the same results three rows later."""
    H, HQ, T, g = 2, 8, 16, torch.Generator().manual_seed(3)
    b, kv = kh.Batch(lengths, T, 2), handle(fmt, H, T)
    q, k, v = (bf(torch.randn(b.n + 3, h * 128, generator=g)) for h in (HQ, H, H))
    found = []
    for shift in (0, 3):
        c = kh.Batch(lengths, T, 2)
        c.starts, c.n_tokens = (c.starts + shift).astype(np.int32), b.n + shift
        qd, kd, vd = (x[3 - shift:].cuda() for x in (q, k, v))
        pk, pv = pools(fmt, b.pool_pages, H, T, 0.5)
        q_rot, out, k2, v2 = (torch.full_like(x, 9.0) for x in (qd, qd, kd, vd))
        lse = torch.full((c.n_tokens, HQ), 9.0, device="cuda")
        cache, batch = tdk.kv_cache(pk, pv, b.pool_pages), c.struct(tdk)
        need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, HQ)
        space = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(kd, vd, H * 128, H * 128, q=qd, q_stride=HQ * 128, n_q_heads=HQ, q_out=q_rot, q_out_stride=HQ * 128), stream())
        tdk.tdk_kv_attend(kv, cache, batch, tdk.kv_attend_io(q_rot, HQ * 128, HQ, 0.1, out, HQ * 128, lse, space, need), stream())
        tdk.tdk_kv_read(kv, cache, batch, tdk.kv_rows(k2, v2, H * 128, H * 128), stream())
        torch.cuda.synchronize()
        for x in (q_rot, out, k2, v2, lse):
            assert (x[:shift] == 9.0).all()
        found.append([bits(x[shift:]) for x in (q_rot, out, k2, v2)] + [lse[shift:].cpu().view(torch.int32)] + [p.cpu().view(torch.uint8) for p in (pk, pv)])
    assert all(torch.equal(x, y) for x, y in zip(*found))


def test_one_handle_from_several_threads():
    """Four host threads, a stream and a workspace each, one handle: each thread's results as if alone."""
    H, HQ, T = 2, 8, 16
    kv = handle(tdk.KV_BF16, H, T)
    jobs = []
    for i, lengths in enumerate([[(900, 1), (3, 1)], [(40, 70)], [(2500, 3)], [(10, 1)] * 30]):
        g, b = torch.Generator().manual_seed(i), kh.Batch(lengths, T, i)
        pk, pv = (bf(torch.randn(b.pool_pages, T, H, 128, generator=g)).cuda() for _ in range(2))
        q, out, lse = bf(torch.randn(b.n, HQ * 128, generator=g)).cuda(), torch.zeros(b.n, HQ * 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.n, HQ, device="cuda")
        batch = b.struct(tdk)
        need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, HQ)
        space = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
        io = tdk.kv_attend_io(q, HQ * 128, HQ, 0.1, out, HQ * 128, lse, space, need)
        cache, st = tdk.kv_cache(pk, pv, b.pool_pages), torch.cuda.Stream()
        tdk.tdk_kv_attend(kv, cache, batch, io, stream())
        torch.cuda.synchronize()
        want = bits(out)
        out.zero_()
        jobs.append(dict(cache=cache, batch=batch, io=io, st=st, out=out, want=want, keep=(b, pk, pv, q, lse, space)))
    torch.cuda.synchronize()
    errors = []

    def work(j):
        try:
            for _ in range(20):
                tdk.tdk_kv_attend(kv, j["cache"], j["batch"], j["io"], j["st"].cuda_stream)
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors and all(torch.equal(bits(j["out"]), j["want"]) for j in jobs)
