"""Static check of the generated code of the kernels around the attention (CPU only: hipcc cross-compiles to assembly).

No kernel may keep registers in scratch, but for two of a norm kernel that has one piece more than fits five workgroups a compute unit.
matmul_kernel waits for the copies that it issued before the stores of a whole tile by counting
what was issued behind them, so the stores have to be as many as it counts: one of 16 bytes for each 16 bytes of a lane's share."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("isa")
    running = []
    for name in ("jenga_norm", "jenga_matmul", "jenga_rotary"):
        path = str(out / (name + ".s"))
        running.append((path, subprocess.Popen(
            ["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-S", "--cuda-device-only", "-o", path,
             os.path.join(CSRC, name + ".hip")], stderr=subprocess.PIPE, text=True)))
    for path, process in running:
        err = process.communicate()[1]
        assert process.returncode == 0, err[-3000:]
    return {os.path.basename(path)[:-2]: open(path).read() for path, _ in running}


def test_nothing_in_scratch(listings):
    for name, text in listings.items():
        kernels = [k for k in text[text.index("amdhsa.kernels:"):].split("\n  - ")[1:] if ".vgpr_spill_count" in k]
        assert len(kernels) >= 10, name
        for k in kernels:
            symbol = re.search(r"\.name:\s+(\S+)", k).group(1)
            for what, most in (("vgpr_spill_count", 2), ("private_segment_fixed_size", 12)):
                value = int(re.search(r"\.%s:\s+(\d+)" % what, k).group(1))
                assert value <= (most if name == "jenga_norm" else 0), (name, symbol, what, value)


def test_stores_of_a_whole_tile(listings):
    text, checked = listings["jenga_matmul"], 0
    for m in re.finditer(r"^(_Z\w*matmul_kernelI(\w+?)Lb[01]ELi(\d+)ELi(\d+)ELi(\d+)E\w*):.*?^\.Lfunc_end", text, re.S | re.M):
        size = 4 if m.group(2) == "f" else 2
        rows, cols, stages = (int(m.group(i)) for i in (3, 4, 5))
        pitch, stage = cols // 2 * size, (rows + cols) * 128
        behind = max((stages - 1) * stage, 4 * 32 * pitch)
        at_once = min(behind // 4 // pitch // 32 * 32, rows // 2)     # rows of a wavefront in LDS at a time
        stores = rows // 2 // (64 // (pitch // 16))
        # those of a whole tile, and one in the loop over the rows of a partial one for each time
        assert len(re.findall(r"global_store_dwordx4 [^\n]* nt", m.group(0))) == stores + rows // 2 // at_once, m.group(1)
        assert not re.findall(r"global_store_dwordx[23] ", m.group(0)), m.group(1)
        checked += 1
    assert checked >= 6
