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


GRID, D, DIMS = (2, 4, 5), 8, (2, 2, 4)


def _in_place(batch, tokens, heads, starts, strides):
    """One or two tensors turned in place, `starts` elements behind A."""
    return GRID, D, DIMS, batch, tokens, [(A + 2 * s, A + 2 * s, heads, strides, strides) for s in starts]


# Q and K as columns of one projection [batch, tokens, 3, heads, D], from one token of each sequence on; head by head
# [batch, 3, heads, tokens, D]; heads of Q and K in turn.
@pytest.mark.parametrize("batch,tokens", [(1, 1), (2, 1), (7, 1), (1, 2), (2, 2), (3, 33)])
def test_interleaved_tensors_are_apart(driver, batch, tokens):
    heads = 3
    row = heads * D
    for strides, k in (((tokens * 3 * row, 3 * row, D), row), ((tokens * 3 * row, 3 * row, D), 2 * row),
                       ((3 * heads * tokens * D, D, tokens * D), heads * tokens * D),
                       ((tokens * 2 * row, 2 * row, 2 * D), D), ((D, 2 * batch * D, 2 * tokens * batch * D), batch * D),
                       ((row, 2 * batch * row, D), batch * row)):
        assert _statuses(driver, [_in_place(batch, tokens, heads, (0, k), strides), _in_place(batch, tokens, heads, (k, 0), strides)]) == \
            [OK, OK], strides
        # where they do share something: half of a head, and the next heads' or rows'
        bad = [_in_place(batch, tokens, heads, (0, k + D // 2), strides)] if k == D else [_in_place(batch, tokens, heads, (0, D // 2), strides)]
        assert _statuses(driver, bad) == [EINVAL], strides


def _places(start, batch, tokens, heads, strides):
    return {start + b * strides[0] + n * strides[1] + h * strides[2] + c
            for b in range(batch) for n in range(tokens) for h in range(heads) for c in range(D)}


# Small layouts at random: none that shares an element with the other is taken, and of two with the same strides each that is apart is.
def test_random_layouts(driver):
    import random
    rng = random.Random(5)
    calls, want = [], []
    while len(calls) < 4000:
        batch, tokens, heads = [rng.choice([1, 1, 2, 3]) for _ in range(3)]
        order, strides, reach = rng.sample(range(3), 3), [0, 0, 0], D
        for i in order:
            strides[i] = reach * rng.choice([1, 1, 2, 3]) + rng.choice([0, 0, 1, D])
            reach = strides[i] * (batch, tokens, heads)[i]
        k = rng.randrange(0, reach + D) if rng.random() < 0.5 else rng.choice(strides)
        heads_k = rng.choice([heads, heads, 1, 2])
        other = [s * rng.choice([1, 1, 1, 2]) for s in strides] if rng.random() < 0.2 else strides
        apart = not _places(0, batch, tokens, heads, strides) & _places(k, batch, tokens, heads_k, other)
        own = _places(k, batch, tokens, heads_k, other)
        if len(own) < batch * tokens * heads_k * D:
            continue
        calls.append((GRID, D, DIMS, batch, tokens, [(A, A, heads, strides, strides), (A + 2 * k, A + 2 * k, heads_k, other, other)]))
        want.append((apart, other == strides))
    taken = 0
    for call, (apart, same), status in zip(calls, want, _statuses(driver, calls)):
        if not apart:
            assert status == EINVAL, call
        elif same:
            assert status == OK, call
            taken += 1
    assert taken > 500
