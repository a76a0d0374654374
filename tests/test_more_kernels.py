"""Kernels of the 8-bit pages, of the prompts' attention and of the rotation, as they are built: registers, scratch, and who uses M0."""
import os
import re
import subprocess

import pytest

from paper_2604_03143_amd import _build
from test_kernel_resources import forms, kernels, waves_per_simd      # noqa: F401  (kernels: the fixture)


def test_no_scratch_and_the_residency_that_calls_are_cut_for(kernels):      # noqa: F811
    """Two workgroups of four wavefronts per compute unit."""
    some = {**dict(forms(kernels, kv8_attend_rows={})), **{k: v for k, v in kernels.items() if k in ("tdk_kv8_attend_tile_kernel", "tdk_prompt_attend_kernel")}}
    assert len(some) == 2 + 2
    for name, (regs, scratch) in some.items():
        assert waves_per_simd(regs) >= 2 and not scratch, name


def test_rows_have_no_scratch(kernels):      # noqa: F811
    some = dict(forms(kernels, kv8_read={}, kv_rotate={}, kv_append_rope={}))
    assert len(some) == 2 + 3 + 6
    assert not {k: v for k, v in some.items() if v[1]}


@pytest.mark.parametrize("source", ["tdk_prompt_attend.hip", "tdk_kv8.hip"])
def test_only_the_direct_loads_use_m0(source, tmp_path):
    """The loads straight into LDS set M0 in inline assembly, which the compiler does not see."""
    out, src = str(tmp_path / "a.s"), os.path.join(_build.CSRC, source)
    cmd = [a for a in _build.hipcc_command(out, extra=["--cuda-device-only", "-S"]) if a not in _build.SOURCES and a not in ("-shared", "-fPIC")]
    subprocess.run([*cmd, src], check=True, capture_output=True, timeout=300)
    inside, own, others = False, 0, []
    for line in open(out):
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
        elif re.search(r"\bm0\b", line.split(";")[0]):
            own += inside
            if not inside:
                others.append(line.strip())
    assert not others and (own > 0) == (source == "tdk_prompt_attend.hip"), (own, others[:5])
