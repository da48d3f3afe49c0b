"""CPU tests of what jenga_rotary takes and refuses, by its argument checks alone, built without the library's kernels."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")
OK, EINVAL, EUNSUPPORTED = 0, -1, -2
BF16 = 0
A = 1 << 20          # far behind the table


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("rotary_args") / "host_operators")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(ROOT, "tests", "host_operators_main.cpp"),
           os.path.join(CSRC, "jenga_plan.cpp"), os.path.join(CSRC, "jenga_host.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


def _statuses(driver, calls):
    """calls: (grid, head_dim, dims, batch, tokens, tensors); a tensor: (src, dst, heads, strides of src, strides of dst)."""
    lines = []
    for grid, head_dim, dims, batch, tokens, tensors in calls:
        line = [*grid, head_dim, *dims, BF16, batch, tokens, len(tensors)]
        for src, dst, heads, s, d in tensors:
            line += [src, dst, heads, *s, *d]
        lines.append(" ".join(str(x) for x in line))
    r = subprocess.run([driver], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    got = [int(x) for x in r.stdout.split()]
    assert len(got) == len(calls)
    return got


# Places in the table are 32-bit numbers in the kernels: pairs of all cells and axes together stay below 2^31 - 1024.
@pytest.mark.parametrize("grid,head_dim,dims,status", [
    ((1 << 24, 1, 1), 256, (254, 0, 0), OK), ((1 << 24, 1, 1), 256, (256, 0, 0), EUNSUPPORTED),
    (((1 << 24) - 8, 1, 1), 256, (256, 0, 0), OK), (((1 << 24) - 7, 1, 1), 256, (256, 0, 0), EUNSUPPORTED),
    ((1 << 23, 1, 1), 1024, (1024, 0, 0), EUNSUPPORTED), ((1 << 22, 1, 1), 1024, (1024, 0, 0), EUNSUPPORTED),
    ((1, 1 << 22, 4), 1024, (0, 1024, 0), EUNSUPPORTED), ((1, 4, 1 << 22), 1024, (2, 2, 1020), OK),
    ((1, 1, 1 << 24), 512, (0, 0, 512), EUNSUPPORTED), ((1 << 12, 1 << 12, 1), 1024, (512, 512, 0), OK)])
def test_tables_past_32_bits(driver, grid, head_dim, dims, status):
    tensor = (4 * A, 12 * A, 1, (0, head_dim, head_dim), (0, head_dim, head_dim))
    for tokens in (0, 1):
        # one token that lies behind the largest table that is taken
        moved = (tensor[0] + (1 << 40), tensor[1] + (1 << 40)) + tensor[2:]
        assert _statuses(driver, [(grid, head_dim, dims, 1, tokens, [moved])]) == [status]


@pytest.mark.parametrize("grid,head_dim,dims", [((1 << 24, 1, 1), 256, (256, 0, 0)), ((1 << 23, 1, 1), 1024, (1024, 0, 0))])
def test_the_library_refuses_them(grid, head_dim, dims):
    import ctypes
    import paper_2505_16864_amd as J
    cfg, list_ = J.make_rotary(*grid, head_dim, dims), (J.jenga_rotary_tensor * 1)()
    for n, v in dict(src=4 * A, dst=12 * A, src_token=head_dim, src_head=head_dim, dst_token=head_dim, dst_head=head_dim, heads=1).items():
        setattr(list_[0], n, v)
    assert J.raw().jenga_rotary(ctypes.byref(cfg), None, None, A, list_, 1, 1, 0, None) == EUNSUPPORTED   # no tokens: nothing to launch
