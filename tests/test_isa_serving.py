"""The serving kernels as the compiler emits them (no GPU needed: hipcc cross-compiles): no instance saves registers to memory but those named."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2501_08071_amd import build as B


@pytest.mark.parametrize("src,kernels,but", [("attn_paged_gfx950.hip", 80, ()), ("kv_append_gfx950.hip", 6, ()),
                                             # 1024 threads a row of odd length to 8 bits: rows past 16384 elements, a few words a thread
                                             ("residual_norm_gfx950.hip", 40, ("Lb1ELi1024ELi4ELb1E",))])
def test_registers_are_enough(src, kernels, but, tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "k.s")
    cmd = [B.HIPCC, *[f for f in B.FLAGS if f != "-fPIC"], "--cuda-device-only", "-S", "-x", "hip", os.path.join(B.CSRC, src), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    sizes = re.findall(r"\.name:\s+(\S*kernel\S*)\n.*?\.private_segment_fixed_size:\s+(\d+)", open(out).read(), flags=re.S)
    assert len(sizes) >= kernels, len(sizes)
    assert not [s for s in sizes if s[1] != "0" and not any(b in s[0] for b in but)]


def test_no_instance_of_the_prefix_kernel_is_out_of_reach():
    """The pass over a prefix has eight wavefronts a workgroup at 16 and at 32 rows (the launch's rule): two types, three head dimensions, two heights,
    and the 128-row kernel."""
    nm = shutil.which("nm")
    if nm is None or not os.path.exists(B.LIB):
        pytest.skip("no nm, or no library")
    names = subprocess.run([nm, "-C", B.LIB], capture_output=True, text=True).stdout
    assert len(set(re.findall(r"attn_paged_prefix_kernel<[^>]*>", names))) == 12
    assert len(set(re.findall(r"attn_paged_wide_prefix_kernel<[^>]*>", names))) == 6
