"""CPU tests of the rule that says which kernel a product takes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("tiles") / "host_operators")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                        os.path.join(ROOT, "tests", "host_operators_main.cpp"), os.path.join(CSRC, "jenga_plan.cpp"),
                        os.path.join(CSRC, "jenga_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def of(sizes):
        """[(m, n, out)] -> [(rows, bm, bn, stages, workgroups a compute unit)]"""
        lines = "".join("%d %d %d\n" % (m, n, out == "f32") for m, n, out in sizes)
        r = subprocess.run([exe, "tiles"], input=lines, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return [tuple(int(x) for x in line.split()) for line in r.stdout.strip().split("\n")]

    return of


# Sizes at which both kinds of tiles were timed: the faster one is taken, but for short k.
@pytest.mark.parametrize("m,n,bm", [
    (1500, 5120, 128), (2048, 5120, 256), (3000, 5120, 256), (4096, 5120, 128), (4352, 5120, 128), (4864, 5120, 128), (4096, 4608, 128),
    (3584, 5632, 128), (8000, 3000, 128), (4500, 4700, 128), (6144, 3840, 128), (2400, 9216, 128), (5120, 5120, 256), (5632, 5632, 256),
    (9000, 4000, 256), (7000, 5000, 256), (9216, 5120, 256), (6700, 7000, 256), (12288, 5120, 256), (33272, 15360, 256), (8192, 8192, 256)])
def test_large_tiles_where_they_were_faster(tiles, m, n, bm):
    assert tiles([(m, n, "bf16")])[0][1] == bm
    assert tiles([(m, n, "f32")])[0][1] == 128


# The sizes that the GPU tests multiply reach every kernel that the rule can name, several tiles a workgroup among them.
def test_tested_sizes_reach_every_kernel(tiles):
    import random
    from matmul_sizes import CASES, SIZES
    at_once = {}
    for (kernel, m, n, _, out), got in zip(CASES, tiles([(m, n, out) for _, m, n, _, out in CASES])):
        assert got[:4] == kernel, (m, n, out)
        if kernel[1]:
            at_once.setdefault((kernel, out), []).append(-(-m // kernel[1]) * -(-n // kernel[2]) / (256 * got[4]))
    for key, rounds in at_once.items():
        assert min(rounds) <= 1 and (key[0][3] == 4 or max(rounds) > 1.5), key
    rng = random.Random(1)
    drawn = [(int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 15)), rng.choice(["bf16", "f32"])) for _ in range(20000)]
    for size, got in zip(drawn, tiles(drawn)):
        assert got[:4] in SIZES and (got[1] != 256 or size[2] != "f32"), size
