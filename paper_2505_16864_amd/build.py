"""Builds libjenga.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
import os
import subprocess
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libjenga.so")
SOURCES = ["jenga_plan.cpp", "jenga_host.cpp", "jenga_permute.hip", "jenga_select.hip", "jenga_attn.hip", "jenga_prores.hip",
           "jenga_norm.hip", "jenga_matmul.hip", "jenga_rotary.hip", "jenga_rms.hip", "jenga_mx.hip", "jenga_dense.hip", "jenga_capi.hip"]


def build_library(verbose=False):
    """Compile every source for gfx950, a compiler each at the same time, and link libjenga.so; raises on failure."""
    flags = ["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC",
             # packed-FP32 VALU forms stay off for all device code
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
    with tempfile.TemporaryDirectory() as objects:
        running = []
        for source in SOURCES:
            to = os.path.join(objects, source + ".o")
            running.append((to, subprocess.Popen(flags + ["-c", os.path.join(CSRC, source), "-o", to], stdout=subprocess.PIPE,
                                                 stderr=subprocess.STDOUT, text=True)))
        failed = False
        for _, process in running:
            said = process.communicate()[0]
            failed = failed or process.returncode != 0
            if verbose or process.returncode != 0:
                print("\n".join(l for l in said.splitlines() if "not a recognized feature" not in l))
        if failed:
            raise RuntimeError("hipcc failed building libjenga.so")
        res = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC"] + [to for to, _ in running] + ["-o", LIB], capture_output=True, text=True)
        if res.returncode != 0:
            print(res.stderr)
            raise RuntimeError("hipcc failed linking libjenga.so")
    return LIB


def build_bench_probe():
    """bench.py's MFMA-only yardstick: its own shared object beside bench.py, not part of the library."""
    src = os.path.join(ROOT, "bench_mfma_probe.hip")
    out = os.path.join(ROOT, "bench_mfma_probe.so")
    cmd = ["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", src, "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        print(res.stderr)
        raise RuntimeError("hipcc failed building bench_mfma_probe.so")
    return out


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_bench_probe())
