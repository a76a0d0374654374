"""tdk_kv_append without queries and tdk_kv_read, up to four KV heads: a wavefront has all of a token, whether the call is small or large."""
import numpy as np
import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk
from test_gpu_kv import FORMATS, bf, bits, handle, pools, stream

pytestmark = pytest.mark.gpu


@FORMATS
@pytest.mark.parametrize("H", [1, 3, 4])
@pytest.mark.parametrize("lengths", [[(7, 1), (0, 2), (40, 0)], [(3, 2045), (9, 3)], [(3, 2046), (9, 3)]])
def test_append_and_read_on_both_sides_of_the_line(fmt, H, lengths):
    """2048 tokens are few on 256 compute units, 2049 are many."""
    T, g = 16, torch.Generator().manual_seed(2)
    b = kh.Batch(lengths, T, 4, pad_tokens=0)
    k, v = (bf(torch.randn(b.n, H * 128, generator=g)) for _ in range(2))
    kd, vd, kv = k.cuda(), v.cuda(), handle(fmt, H, T)
    pk, pv = pools(fmt, b.pool_pages, H, T, 7.0)
    cache, batch = tdk.kv_cache(pk, pv, b.pool_pages), b.struct(tdk)
    tdk.tdk_kv_append(kv, cache, batch, tdk.kv_rows(kd, vd, H * 128, H * 128), stream())
    k2, v2 = (torch.full((b.n, H * 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tdk.tdk_kv_read(kv, cache, batch, tdk.kv_rows(k2, v2, H * 128, H * 128), stream())
    torch.cuda.synchronize()
    pos = [p for _, p in b.positions()]
    rows = torch.from_numpy(kh.rotate(k.float().numpy().reshape(b.n, H, 128), pos, 1e6, False)), v.float().reshape(b.n, H, 128)
    for got, pool, x in ((k2, pk, rows[0]), (v2, pv, rows[1])):
        want = bf(x) if fmt == tdk.KV_BF16 else bf(kh.from4(*kh.to4(x)))
        assert torch.equal(bits(got).reshape(b.n, H, 128), bits(want))
        # and nothing else was written
        mark = torch.ones(b.pool_pages, T, dtype=torch.bool)
        for s, p in b.positions():
            mark[b.slot(s, p)] = False
        rest = pool.cpu()
        if fmt == tdk.KV_BF16:
            assert (rest[mark] == 7.0).all()
        else:
            codes, bytes_ = kh.unpack4(rest, T)
            assert (bytes_[mark] == 0x5A).all() and (codes[mark].reshape(-1, 2) == torch.tensor([0xA, 0x5])).all()
    assert np.array_equal(b.d[1].cpu().numpy(), b.lens)
