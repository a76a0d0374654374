"""The bounds that the GPU tests of far scores use: right results pass, zeros and exchanged rows do not (on the CPU, mistakes planted in the wanted results)."""
import pytest
import torch

import far_helpers as fh
import kv_helpers as kh
import prompt_helpers as ph


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("window,sink", [(0, 0), (60, 3)])
def test_shifted(sign, window, sink):
    n = 200
    q, k, v = (x.double() for x in fh.rows(n, 10, n, 2, 3, sign))
    want, lse, mass, big = ph.attend([(n, n)], q, k, v, fh.SCALE, window, sink)
    assert 3982 <= big < 4100 and (lse.abs() * 1.4427 > 4096 + 1000).all()
    tol, ltol = kh.tolerance(want, lse, mass, big, n)
    assert fh.wrong_shifted(want.to(torch.bfloat16).double(), want, tol) == 0 and ltol.max() < 0.05
    for bad in fh.mistaken(want):
        assert fh.wrong_shifted(bad, want, tol) > 0.4 * want.numel()


@pytest.mark.parametrize("scale", [2.0 ** 20, -2.0 ** 40])
def test_steep(scale):
    n = 120
    q, k, v = (x.double() for x in fh.rows(n, 10, n, 2, 4))
    bounds = fh.steep_all(q, k, v, scale, [range(i + 1) for i in range(n)])
    assert bounds[0].double().mean() > 0.95
    want, _, _, _ = ph.attend([(n, n)], q, k, v, scale)
    assert fh.wrong_steep(want.to(torch.bfloat16).double(), bounds) == 0
    for bad in fh.mistaken(want):
        assert fh.wrong_steep(bad, bounds) > 0.5 * want.numel()
