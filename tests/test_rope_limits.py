"""tdk_kv_rotate: as many tokens as one launch holds, 2^32 threads of which a token takes 256 at most, whatever its heads."""
import pytest
import torch

from paper_2604_03143_amd import tdk
from test_kv_args import batch, refused
from test_rope_args import io, lib, make      # noqa: F401  (lib: the fixture)

MOST = (1 << 24) - 1


@pytest.mark.skipif(torch.cuda.is_available(), reason="a machine without a GPU is meant")
@pytest.mark.parametrize("n_q_heads", [1, 8, 40, 512])
@pytest.mark.parametrize("n_tokens", [1 << 22, (1 << 22) + 1, MOST])
def test_tokens_up_to_the_limit_get_as_far_as_the_device(n_q_heads, n_tokens):
    wide = n_q_heads * 128
    refused(lambda: tdk.tdk_kv_rotate(make(), batch(n_tokens=n_tokens), io(n_q_heads=n_q_heads, q_stride=wide, q_out_stride=wide)), say="device")


@pytest.mark.parametrize("n_q_heads", [1, 40])
def test_more_are_refused(n_q_heads):
    wide = n_q_heads * 128
    refused(lambda: tdk.tdk_kv_rotate(make(), batch(n_tokens=MOST + 1), io(n_q_heads=n_q_heads, q_stride=wide, q_out_stride=wide)), tdk.ERR_UNSUPPORTED, "launch")
