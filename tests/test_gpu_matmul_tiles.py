"""jenga_matmul through each of its kernels, several tiles a workgroup among them, against float64; tolerances as in test_gpu_matmul.py:
16-bit results are off by their rounding and 8 * 2^-13 of the sum of the products' magnitudes at most (2^-12 of the norm in the root mean
square), float32 results by k + 8 additions of 2^-24 (2^-19)."""
import pytest
import torch

from matmul_sizes import CASES, ROWS_32, SIZES, TILES_128, TILES_256
from operator_util import TYPES, U32, check, half_step, held_values, randn

pytestmark = pytest.mark.gpu


def _quantized(x, block_rows):
    import paper_2505_16864_amd as J
    rows, cols = x.shape
    q = torch.empty((rows, J.padded_columns(cols)), dtype=torch.uint8, device="cuda:0")
    scale = torch.empty((-(-rows // block_rows), J.scale_columns(cols)), dtype=torch.uint8, device="cuda:0")
    J.jenga_quantize(x, q, scale, block_rows)
    return q, scale


def _operands(m, n, k, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    x = torch.randn((m, k), generator=gen, device="cuda:0") * torch.exp(0.5 * torch.randn((m, 1), generator=gen, device="cuda:0"))
    w = torch.randn((n, k), generator=gen, device="cuda:0") * torch.exp(0.5 * torch.randn((n, 1), generator=gen, device="cuda:0"))
    return _quantized(x, 1) + _quantized(w, 128)


def _held(q, scale, block_rows):
    return held_values(q.view(torch.float8_e4m3fn), scale, block_rows).cuda()


# The result with and without a bias, next to each other and among other columns.
@pytest.mark.parametrize("kernel,m,n,k,out", CASES)
def test_every_kernel(kernel, m, n, k, out):
    import paper_2505_16864_amd as J
    a, a_scale, b, b_scale = _operands(m, n, k, m + n + k)
    dtype = TYPES[out]
    A, B = _held(a, a_scale, 1), _held(b, b_scale, 128)
    product, size = A @ B.t(), A.abs() @ B.abs().t()
    for bias in (None, randn(3, n).float()):
        room = torch.full((m, n + 13), 7.0, dtype=dtype, device="cuda:0")
        alone = torch.full((m, n), 7.0, dtype=dtype, device="cuda:0")
        for got in (alone, room[:, 5:5 + n]):
            J.jenga_matmul(a, a_scale, b, b_scale, got, bias if bias is None else bias.cuda())
        torch.cuda.synchronize()
        assert torch.equal(room[:, 5:5 + n], alone) and bool((room[:, :5] == 7).all()) and bool((room[:, 5 + n:] == 7).all())
        want = (product if bias is None else product + bias.cuda().double()).cpu()
        whole = (size if bias is None else size + bias.cuda().double().abs()).cpu()
        rms = float((alone.cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt())
        if out == "f32":
            check(alone, want, U32 * (k + 8) * whole, "%s" % (kernel,))
            assert rms <= 2.0 ** -19, rms
        else:
            least = 2.0 ** -25 if out == "f16" else 0.0
            check(alone, want, half_step(dtype) * want.abs() * 1.01 + 8 * 2.0 ** -13 * whole + least, "%s" % (kernel,))
            assert rms <= half_step(dtype) + 2.0 ** -12, rms


# One size of each kernel in one graph, the several tiles a workgroup of each result type among them; every replay against the eager result,
# with eager work of the same calls between the replays.
def test_every_kernel_in_a_graph():
    import paper_2505_16864_amd as J
    sizes = [(*SIZES[kernel][0], out) for kernel, out in zip(SIZES, ("bf16", "f32", "f16", "f32", "bf16", "f16"))]
    sizes += [(*SIZES[TILES_128][1], out) for out in ("bf16", "f16", "f32")] + [(*SIZES[TILES_256][1], "bf16"), (*SIZES[ROWS_32][0], "bf16")]
    work = []
    for i, (m, n, k, out) in enumerate(sizes):
        b, b_scale = _quantized(randn(30 + i, n, k).float().cuda(), 128)
        gen = torch.Generator(device="cuda:0").manual_seed(i)
        x = [torch.randn((m, k), generator=gen, device="cuda:0") for _ in range(3)]
        a, a_scale = _quantized(x[0], 1)
        work.append((x, x[0].clone(), a, a_scale, b, b_scale, torch.empty((m, n), dtype=TYPES[out], device="cuda:0")))

    def run(which=None):
        for x, now, a, a_scale, b, b_scale, out in work:
            J.jenga_quantize(now if which is None else x[which], a, a_scale)
            J.jenga_matmul(a, a_scale, b, b_scale, out)

    want = []
    for i in range(3):
        run(i)
        want.append([w[-1].clone() for w in work])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in (1, 2, 0, 2):
        for w in work:
            w[1].copy_(w[0][i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(w[-1], t) for w, t in zip(work, want[i])), i
        run((i + 1) % 3)
        torch.cuda.synchronize()
        assert all(torch.equal(w[-1], t) for w, t in zip(work, want[(i + 1) % 3])), i


# What the gradients rest on: the transpose of a matrix in blocks of 128 x 128 holds the same values, as the kernel quantises both.
@pytest.mark.parametrize("rows,cols", [(1, 1), (127, 130), (128, 512), (200, 300), (384, 256), (700, 1000)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_transposes_hold_the_same_values(rows, cols, dtype):
    w = (randn(rows + cols, rows, cols) * torch.exp(2 * randn(2, rows, 1))).to(TYPES[dtype]).cuda()
    held, turned = _held(*_quantized(w, 128), 128), _held(*_quantized(w.t().contiguous(), 128), 128)
    assert torch.equal(held[:, :cols], turned[:, :rows].t()) and not held[:, cols:].any() and not turned[:, rows:].any()
    # and they are w to half a step of e4m3, or half of the smallest one, 2^-10 of a unit below 2^-7 of the largest value
    off = (held[:, :cols] - w.double()).abs()
    assert bool((off <= 2.0 ** -4 * w.double().abs() + 2.0 ** -17 * w.double().abs().max()).all())
