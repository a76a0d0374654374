"""tdk_kv_attend at scales of every size, and scores of every size."""
import math

import numpy as np
import pytest
import torch

import kv_helpers as kh
from paper_2604_03143_amd import tdk
from test_gpu_kv import FORMATS, bf
from test_gpu_kv_values import close, run

pytestmark = pytest.mark.gpu


def whole(b, fmt, H, group, seed, size=1.0):
    """K and Q of small whole numbers (times `size`, a power of two): every score is exact in 32 bits."""
    g = torch.Generator().manual_seed(seed)
    k = bf(torch.randint(-3, 4, (b.pool_pages, b.T, H, 128), generator=g).double() * size)
    v = bf(torch.randn(b.pool_pages, b.T, H, 128, generator=g))
    q = bf(torch.randint(-3, 4, (b.n, H * group, 128), generator=g).double() * size)
    if fmt == tdk.KV_BF16:
        return k, v, q, k.double(), v.double()
    packed = [kh.to4(x.float()) for x in (k, v)]
    assert torch.equal(kh.from4(*packed[0]), k.double())                  # (whole numbers up to 3 are 4-bit values of any block they stand in)
    return *(kh.pack4(*x, b.T) for x in packed), q, k.double(), kh.from4(*packed[1])


SCALE_LENGTHS = pytest.mark.parametrize("lengths", [[(50, 1), (20, 3), (0, 1)], [(5000, 1)], [(0, 70), (90, 40)], [(2500, 9)], [(1500, 60)]])


def check_scale(fmt, lengths, scale, size=1.0, kw={}, join=False):
    H, group, T = 2, 4, 16
    b = kh.Batch(lengths, T, 3)
    dk, dv, q, k, v = whole(b, fmt, H, group, 5, size)
    part = (None, None)
    if join:
        g = torch.Generator().manual_seed(6)
        part = (torch.randn(b.n, H * group, 128, generator=g), torch.randn(b.n, H * group, generator=g))
    want, wlse, mass, _ = kh.attend(b, k, v, q.double(), float(np.float32(scale)), **kw, part_out=None if part[0] is None else part[0].double(),
                                    part_lse=None if part[1] is None else part[1].double())
    got, glse = run(b, fmt, H, group, dk, dv, q, scale, **kw, part=part)
    return want, wlse, mass, got, glse, max(h + n for h, n in lengths)


@FORMATS
@SCALE_LENGTHS
@pytest.mark.parametrize("scale", [1.0e6, 1.0e8, 1.0e9, -1.0e9, 1.0e30, 2.0 ** 127])
@pytest.mark.parametrize("kw,join", [({}, False), (dict(window=37, sink=5), True)])
def test_large_scales(fmt, lengths, scale, kw, join):
    """Only the largest scores of a row count, equally where several are equal.  Scores are whole numbers, exact; so are the weights then,
    one and zero: the sums over n tokens add 2^-24 a step, the division one more, the output 2^-8.  The logarithm is the scaled maximum
    (2^-24 of it; infinite where fp32 has no such number) plus that of a count (two steps of fp32)."""
    want, wlse, mass, got, glse, n = check_scale(fmt, lengths, scale, kw=kw, join=join)
    close(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -24 * (n + 4) * mass)
    close(glse, wlse.float().double(), 2.0 ** -22 * (wlse.abs() + 16))


@FORMATS
@pytest.mark.parametrize("q_size", [2.0 ** 20, 2.0 ** 50])
def test_large_scores_at_an_ordinary_scale(fmt, q_size):
    """The same of queries and keys that are large themselves."""
    for lengths in ([(50, 1), (20, 3), (0, 1)], [(5000, 1)], [(0, 70), (90, 40)]):
        want, wlse, mass, got, glse, n = check_scale(fmt, lengths, 1 / math.sqrt(128), size=q_size)
        close(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -24 * (n + 4) * mass)
        close(glse, wlse, 2.0 ** -22 * (wlse.abs() + 16))


@FORMATS
@SCALE_LENGTHS
@pytest.mark.parametrize("scale", [0.0, -0.0, 1.0e-45])
def test_scales_that_make_all_weights_equal(fmt, lengths, scale):
    """Scores of up to 2^122: times zero they are zero, times 2^-149 less than 2^-26 (the weights differ by less than a step of fp32)."""
    want, wlse, mass, got, glse, n = check_scale(fmt, lengths, scale, size=2.0 ** 56)
    close(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -24 * (n + 6) * mass + 2.0 ** -8 * 2.0 ** -24)
    close(glse, wlse, torch.full_like(wlse, 2.0 ** -22 * 16))


@FORMATS
@SCALE_LENGTHS
@pytest.mark.parametrize("scale", [1.0e-36, -1.0e-36, 3.0e-37])
def test_small_scales_of_large_scores(fmt, lengths, scale):
    """Scales far below one are taken as they are: scores of up to 2^122 become ordinary ones.  Exact before the scale; the scale's and the
    product's roundings are 2^-22 of an exponent of at most 64, and the weights are rounded to bf16 (2^-8)."""
    want, wlse, mass, got, glse, n = check_scale(fmt, lengths, scale, size=2.0 ** 56)
    e = 2.0 ** -22 * 64 + 2.0 ** -22 + 2.0 ** -24 * n
    close(got, want, 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * e) * 1.01 * mass)
    close(glse, wlse, torch.full_like(wlse, e + 2.0 ** -22 * 66))


@pytest.mark.parametrize("lengths", [[(50, 1), (20, 3)], [(0, 70)], [(3000, 1)]])
@pytest.mark.parametrize("scale", [0.0, 0.1, 1.0e30])
def test_scores_that_are_all_minus_infinity(lengths, scale):
    """Such a row is as one that sees nothing; joined, the other part is all there is."""
    H, group, T = 2, 4, 16
    b, g = kh.Batch(lengths, T, 3), torch.Generator().manual_seed(4)
    k, v = torch.full((b.pool_pages, T, H, 128), -math.inf, dtype=torch.bfloat16), bf(torch.randn(b.pool_pages, T, H, 128, generator=g))
    q = torch.ones(b.n, H * group, 128, dtype=torch.bfloat16)
    out, lse = run(b, tdk.KV_BF16, H, group, k, v, q, scale)
    assert (out == 0).all() and (lse == -math.inf).all()
    part = torch.randn(b.n, H * group, 128, generator=g), torch.randn(b.n, H * group, generator=g)
    out, lse = run(b, tdk.KV_BF16, H, group, k, v, q, scale, part=part)
    close(out, part[0].double(), 2.0 ** -8 * part[0].double().abs())
    close(lse, part[1].double(), torch.zeros(()))


@FORMATS
@SCALE_LENGTHS
@pytest.mark.parametrize("scale", [8.0, 14.0, 20.0, -14.0])
def test_reference_points_on_both_sides_of_two_to_the_twelfth(fmt, lengths, scale):
    """Where the step kernel begins to subtract before it scales.  Scores are exact; a reference point of up to 2^12 in base 2 is rounded by 2^-12 at
    most, twice (product and constant), and sums of two reference points meet: e = 2^-10 of an exponent, and as much for all other roundings.
    (Where the largest weight meets a V of zero, what is left may be 1e-91: weights below 2^-126, the least normal fp32 number, with the 2^12 that
    all are taken lower below 2^-114 of the largest, may vanish; 2^13 tokens of |V| up to 2^3 together no more than 2^-98.)"""
    want, wlse, mass, got, glse, n = check_scale(fmt, lengths, scale)
    e = 2.0 ** -9 + 2.0 ** -24 * n
    close(got, want, 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * e) * 1.01 * mass + 2.0 ** -98)
    close(glse, wlse, e + 2.0 ** -22 * wlse.abs())
