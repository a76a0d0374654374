"""The step kernels of the attention over pages, as they are built."""
from test_kernel_resources import forms, kernels      # noqa: F401  (kernels: the fixture)


def test_step_kernels_have_no_scratch_in_either_format(kernels):      # noqa: F811
    tile = dict(forms(kernels, kv_attend_tile={}))
    assert len(tile) == 2 and not {k: v for k, v in tile.items() if v[1]}
