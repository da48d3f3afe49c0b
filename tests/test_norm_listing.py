"""Static check of the generated code of the layer norm (CPU only: hipcc cross-compiles to assembly): no kernel keeps vector registers in
scratch but norm_kernel of bf16 rows with three pieces of one wavefront, two of them: its registers do not all fit five workgroups a unit."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")


def test_vector_registers_in_scratch(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    path = str(tmp_path / "norm.s")
    r = subprocess.run(["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                        "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-S", "--cuda-device-only", "-o", path,
                        os.path.join(CSRC, "jenga_norm.hip")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    text = open(path).read()
    kernels = [k for k in text[text.index("amdhsa.kernels:"):].split("\n  - ")[1:] if ".vgpr_spill_count" in k]
    number = lambda what, k: int(re.search(r"\.%s:\s+(\d+)" % what, k).group(1))  # noqa: E731
    assert len(kernels) > 100
    spilled = {re.search(r"\.name:\s+(\S+)", k).group(1): number("vgpr_spill_count", k) for k in kernels
               if number("vgpr_spill_count", k) or number("private_segment_fixed_size", k)}
    # norm_kernel<X, X, false, 3, 1> of bf16 (fp16 rows fit)
    assert all(re.search(r"11norm_kernelIDF16bDF16bLb0ELi3ELi1EE", name) and n <= 2 for name, n in spilled.items()), spilled
