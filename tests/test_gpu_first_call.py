"""The first call of a process on each operator is a captured one."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
import paper_2505_16864_amd as J
t = lambda *shape, dtype=torch.bfloat16: torch.ones(shape, dtype=dtype, device="cuda:0")
# h = 2 / sqrt(4 + 1e-6) is off 1 by 1.3e-7, its float32 sums by 80 * 2^-24 at most; a byte of 1 is 0.5 in the even column and 0 in the odd one
x, w, y, total, rstd = t(70, 640), t(640), t(70, 640), t(70, 640), t(70, dtype=torch.float32)
q, s, b, bs, out = t(70, 320, dtype=torch.uint8), t(70, 20, dtype=torch.uint8), t(200, 320, dtype=torch.uint8), t(200, 20, dtype=torch.uint8) * 127, t(70, 200)
dx, dw, room = t(70, 640), t(640, dtype=torch.float32), t(J.jenga_rms_norm_grad_workspace(70, 640), dtype=torch.uint8)
starts, space, o = torch.tensor([0, 30, 70], dtype=torch.int32, device="cuda:0"), t(J.jenga_dense_attn_workspace(70, 70, 2, 5, 5, 128), dtype=torch.uint8), t(70, 5, 128)
h = x.view(70, 5, 128)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    J.jenga_rms_norm(x, y, w, residual=x, total=total, rstd=rstd)
    J.jenga_rms_norm_grad(total, y, dx, w, rstd, dweight=dw, workspace=room)
    J.jenga_quantize_mx(y, q, s)
    J.jenga_matmul_mx(q, s, b, bs, out)
    J.jenga_dense_attn(h, h, h, o, starts, starts, causal=True, workspace=space)
for _ in range(3):
    graph.replay()
    torch.cuda.synchronize()
assert bool((y == 1).all()) and bool((total == 2).all()) and bool((o == 1).all()) and bool(((dw - 70).abs() < 70 * 6e-6).all()) and bool((out == 320 * 0.5).all()), (y, o, dw, out)
print("as eager calls")
"""


def test_first_call_is_captured():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "as eager calls" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
