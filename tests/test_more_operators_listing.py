"""Static check of the generated code of the norm without a mean, the 4-bit products and dense attention (CPU only: hipcc cross-compiles to
assembly): which kernels keep vector registers in scratch, and that the stores of a whole tile of products are as many as the kernel counts."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")
# the few that do, and how many: none in a loop over blocks or steps, but those of float32 products in tiles of 256 x 256
SPILLED = {r"rms_grad_kernelI\w+Li1024ELi2EE": 16, r"rms_grad_kernelIffLi768ELi2EE": 24, r"matmul_mx_kernelI\w+Li256ELi256E": 40,
           r"dense_tiles_kernelI\w+Li128ELb0E": 4}


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("isa")
    running = []
    for name in ("jenga_rms", "jenga_mx", "jenga_dense"):
        path = str(out / (name + ".s"))
        running.append((path, subprocess.Popen(
            ["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-S", "--cuda-device-only", "-o", path,
             os.path.join(CSRC, name + ".hip")], stderr=subprocess.PIPE, text=True)))
    for path, process in running:
        err = process.communicate()[1]
        assert process.returncode == 0, err[-3000:]
    return {os.path.basename(path)[:-2]: open(path).read() for path, _ in running}


def test_vector_registers_in_scratch(listings):
    for name, text in listings.items():
        kernels = [k for k in text[text.index("amdhsa.kernels:"):].split("\n  - ")[1:] if ".vgpr_spill_count" in k]
        assert len(kernels) >= 10, name
        for k in kernels:
            symbol = re.search(r"\.name:\s+(\S+)", k).group(1)
            spilled = int(re.search(r"\.vgpr_spill_count:\s+(\d+)", k).group(1))
            most = max([n for pattern, n in SPILLED.items() if re.search(pattern, symbol)], default=0)
            assert spilled <= most, (symbol, spilled)


def _inner_loops(body):
    """Bodies of the innermost loops of a kernel, by the compiler's own marks."""
    blocks = re.split(r"^\.LBB", body, flags=re.M)
    return [b for b in blocks if "Inner Loop Header" in b[:400]]


def test_no_scratch_in_the_loop_over_blocks(listings):
    checked = 0
    for m in re.finditer(r"^(_Z\w*(?:matmul_mx_kernel|dense_tiles_kernel|dense_rows_kernel)I\w*):.*?^\.Lfunc_end", listings["jenga_mx"] + listings["jenga_dense"],
                         re.S | re.M):
        for block in _inner_loops(m.group(0)):
            if "v_mfma" in block and "matmul_mx_kernelIfLi256" not in m.group(1):
                assert "scratch_" not in block, m.group(1)
                checked += 1
    assert checked >= 10


def test_stores_of_a_whole_tile(listings):
    text, checked = listings["jenga_mx"], 0
    for m in re.finditer(r"^(_Z\w*matmul_mx_kernelI(\w+?)Li(\d+)ELi(\d+)ELi(\d+)E\w*):.*?^\.Lfunc_end", text, re.S | re.M):
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
    assert checked >= 9
