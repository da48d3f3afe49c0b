"""CPU tests of what the host reckons for dense attention without knowing lengths: the work that the device finds from any lengths fits the
launch, the list and the workspace.  The device's rules are written here a second time, in float32 where it has float32."""
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_16864_amd", "csrc")
F = np.float32
NAMES = ("rows", "workgroups", "may_split", "listed", "tiles", "items", "slots", "split_tiles", "bins_at", "items_at", "merge_at", "stat_at", "part_at",
         "workspace")


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("dense") / "host_dense")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(ROOT, "tests", "host_dense_main.cpp"),
                        os.path.join(CSRC, "jenga_plan.cpp"), os.path.join(CSRC, "jenga_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def of(configs):
        r = subprocess.run([exe], input="".join("%d %d %d %d %d %d\n" % c for c in configs), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return [dict(zip(NAMES, map(int, line.split()))) for line in r.stdout.strip().split("\n")]

    return of


def _ceil(a, b):
    return -(-a // b)


def _work(s, q, kv, heads, kv_heads, causal):
    """Tiles, items, slots and cut tiles of a call."""
    group, keys = heads // kv_heads, 64
    tiles = [_ceil(n * group, s["rows"]) for n in q]
    total = sum(tiles)

    def seen(nq, nk, t):            # keys of tile t
        if not causal:
            return nk
        last = min((t * s["rows"] + s["rows"] - 1) // group, nq - 1)
        return max(0, min(nk, last + 1 + nk - nq))

    def chunk_of(steps, longest):
        if not s["may_split"] or total * kv_heads >= 2 * s["workgroups"] or total == 0:
            return 0
        share = F(F(F(steps) * F(kv_heads)) / F(s["workgroups"]))
        rounds = F(_ceil(total * kv_heads, s["workgroups"]))
        if s["rows"] == 16:
            if max(F(longest), F(rounds * F(steps)) / F(total)) <= F(1.15) * share + F(4):
                return 0
            return max(int(np.ceil(F(0.5) * share)), 4)
        return 0 if F(longest) <= F(3) * share + F(8) else max(int(np.ceil(share)), 4)

    def parts(chunk, n):
        return 1 if chunk == 0 else min(64, max(1, _ceil(_ceil(n, keys), chunk)))

    if s["listed"]:
        per_tile = [seen(nq, nk, t) for nq, nk, n in zip(q, kv, tiles) for t in range(n)] if s["may_split"] and total <= 1024 else []
        steps = [_ceil(n, keys) for n in per_tile]
        chunk = chunk_of(sum(steps), max(steps, default=0)) if per_tile else 0
        counts = [parts(chunk, n) for n in per_tile] if chunk else [1] * total
        return total, sum(counts), sum(c for c in counts if c > 1), sum(c > 1 for c in counts)
    steps = [F(0.5) * F(n) * F(_ceil(seen(nq, nk, 0), keys) + _ceil(nk, keys)) if n else F(0) for nq, nk, n in zip(q, kv, tiles)]
    chunk = chunk_of(sum(steps), max([_ceil(nk, keys) for nk, n in zip(kv, tiles) if n], default=0))
    places = sum(n * parts(chunk, nk) for n, nk in zip(tiles, kv))
    return total, places, places if chunk else 0, total if chunk else 0


def _lengths(rng, count, most):
    return [0 if rng.random() < 0.1 else int(round(most ** rng.random())) for _ in range(count)]


@pytest.mark.parametrize("seed", range(40))
def test_work_fits_what_the_host_reckons(shapes, seed):
    rng = random.Random(seed)
    cases = []
    for _ in range(60):
        heads, kv_heads = rng.choice([(1, 1), (2, 2), (5, 1), (6, 3), (12, 12), (32, 8), (40, 8), (40, 40), (64, 1), (96, 96), (3, 1)])
        count, most = rng.choice([1, 2, 3, 7, 16, 40, 64, 65, 100, 300, 1000]), rng.choice([1, 4, 40, 700, 16000])
        kv = _lengths(rng, count, rng.choice([1, 100, 3000, 131072]))
        form = rng.random()
        q = [1] * count if form < 0.3 else kv[:] if form < 0.5 else _lengths(rng, count, most)
        if sum(q) and sum(q) < 200000:
            cases.append((q, kv, heads, kv_heads, rng.choice([64, 128]), rng.random() < 0.5))
    got = shapes([(sum(q), sum(kv), len(q), h, k, d) for q, kv, h, k, d, _ in cases])
    cut = 0
    for s, (q, kv, h, k, d, causal) in zip(got, cases):
        tiles, items, slots, merges = _work(s, q, kv, h, k, causal)
        what = (s, q[:70], kv[:70], h, k, d, causal)
        assert tiles <= s["tiles"] and items <= s["items"] and slots <= s["slots"] and merges <= s["split_tiles"], what
        cut += slots > 0
        assert s["items_at"] - s["bins_at"] >= 4 * (len(q) + 1) and s["merge_at"] - s["items_at"] >= 32 * s["items"], what
        assert s["stat_at"] - s["merge_at"] >= 24 * s["split_tiles"] and s["part_at"] - s["stat_at"] >= 8 * s["slots"] * k * s["rows"], what
        assert s["workspace"] - s["part_at"] >= 4 * s["slots"] * k * s["rows"] * d, what
        assert all(s[n] % 256 == 0 for n in NAMES[8:13])
    assert cut >= 3
