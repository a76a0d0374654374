"""The kernels of the caches that programs append to, as they are built: registers, scratch, and who uses M0."""
import os
import re
import subprocess


from paper_2604_03143_amd import _build
from test_kernel_resources import forms, kernels, waves_per_simd      # noqa: F401  (kernels: the fixture)


def test_kernels_have_the_residency_that_calls_are_cut_for(kernels):      # noqa: F811
    """Two workgroups of four wavefronts per compute unit, three of the 4-bit kernel for up to 16 rows."""
    rows = dict(forms(kernels, kv_attend_rows={}))
    tile = dict(forms(kernels, kv_attend_tile={}))
    assert len(rows) == 3 and len(tile) == 2
    for name, (regs, _) in {**rows, **tile}.items():
        assert waves_per_simd(regs) >= (3 if name == "tdk_kv_attend_rows_kernel<true, 1>" else 2), name


def test_no_scratch_where_loads_are_counted_on(kernels):      # noqa: F811
    """A reload from scratch waits for every load issued before it.  (The 4-bit step kernel keeps a few words there.)"""
    some = dict(forms(kernels, kv_attend_rows={}, kv_attend_tile={0: "false"}, kv_append={}, kv_read={}))
    assert len(some) == 3 + 1 + 4 + 4
    assert not {k: v for k, v in some.items() if v[1]}


def test_only_the_direct_loads_use_m0(tmp_path):
    """As in the spans' attention kernels: the loads straight into LDS set M0 in inline assembly, which the compiler does not see."""
    out, src = str(tmp_path / "kv.s"), os.path.join(_build.CSRC, "tdk_kv.hip")
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
    assert own > 0 and not others, (own, others[:5])
