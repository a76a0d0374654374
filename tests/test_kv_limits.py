"""tdk_kv_*: calls beyond what the kernels count in, refused on the host."""
import os

import pytest

from paper_2604_03143_amd import tdk
from test_kv_args import batch, cache, io, make, refused, rows


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(tdk.LIB_PATH):
        from paper_2604_03143_amd import _build
        _build.build(force=True)
    return tdk.load()


@pytest.mark.parametrize("n_seqs", [(1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 63, (1 << 31) - 1])
def test_too_many_sequences(n_seqs):
    """The search for a token's sequence goes in steps of 64 over 32-bit numbers: from 2^31 - 63 sequences on, their sum wraps."""
    kv = make()
    for f in (lambda: tdk.tdk_kv_append(kv, cache(), batch(n_seqs=n_seqs), rows()), lambda: tdk.tdk_kv_read(kv, cache(), batch(n_seqs=n_seqs), rows()),
              lambda: tdk.tdk_kv_attend(kv, cache(), batch(n_seqs=n_seqs), io())):
        refused(f, tdk.ERR_UNSUPPORTED, "2^30 sequences")


@pytest.mark.parametrize("scale", [1.01 * 2.0 ** 127, -3.4e38])
def test_scales_whose_product_with_a_logarithm_is_beyond_fp32(scale):
    refused(lambda: tdk.tdk_kv_attend(make(), cache(), batch(), io(scale=scale)), say="2^127")
