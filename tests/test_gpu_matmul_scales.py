"""jenga_matmul of blocks whose scales lie anywhere in their byte, against float64.

Tolerances as in test_gpu_matmul.py, and what the header says of the ends of the range.  16-bit results: sums below 2^-126 may be taken as 0,
after each of at most k / 32 steps.  Float32 results: a value below 2^-126 may be taken as 0, so either operand's are off by 2^-126; float32
sums are rounded to multiples of 2^-149."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, held_values, randn

pytestmark = pytest.mark.gpu


def _quantized(x, block_rows):
    import paper_2505_16864_amd as J
    rows, cols = x.shape
    q = torch.empty((rows, J.padded_columns(cols)), dtype=torch.uint8, device="cuda:0")
    scale = torch.empty((-(-rows // block_rows), J.scale_columns(cols)), dtype=torch.uint8, device="cuda:0")
    J.jenga_quantize(x.cuda(), q, scale, block_rows)
    return q, scale


def _check(a, b, k, out):
    import paper_2505_16864_amd as J
    got = torch.empty((a[0].shape[0], b[0].shape[0]), dtype=TYPES[out], device="cuda:0")
    J.jenga_matmul(*a, *b, got)
    torch.cuda.synchronize()
    A, B = held_values(*a, 1), held_values(*b, 128)
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    if out == "f32":
        lost = 2.0 ** -126 * (A.abs().sum(1)[:, None] + B.abs().sum(1)[None] + k * 2.0 ** -126)
        check(got, want, U32 * (k + 8) * size + lost + k * 2.0 ** -149, "float32")
    else:
        check(got, want, half_step(TYPES[out]) * want.abs() * 1.01 + 8 * 2.0 ** -13 * size + (k / 32 + 1) * 2.0 ** -126, out)


# Every operand's blocks at one magnitude: no rows of tiles, small tiles, large ones.
@pytest.mark.parametrize("m,n,k", [(5, 300, 640), (300, 260, 128), (2100, 2300, 384)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("ea,eb", [(-130, 100), (-135, 120), (-126, 20), (-120, 0), (110, -100), (118, -130), (119, 0), (-60, -60), (-70, -70),
                                   (60, 55), (0, -126)])
def test_magnitudes(m, n, k, out, ea, eb):
    a, b = _quantized((randn(1, m, k) * 2.0 ** ea).float(), 1), _quantized((randn(2, n, k) * 2.0 ** eb).float(), 128)
    _check(a, b, k, out)


# Each block at a magnitude of its own, over the whole range of bytes, so that neighbours in a row and in a tile differ by up to 2^200.
@pytest.mark.parametrize("m,n,k", [(9, 300, 1280), (300, 520, 1280), (2100, 2300, 640)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_magnitudes_of_their_own(m, n, k, out):
    gen = torch.Generator().manual_seed(m)
    blocks = k // 128
    ea = torch.randint(-120, 60, (m, blocks), generator=gen).repeat_interleave(128, 1)
    eb = torch.randint(-120, 50, (-(-n // 128), blocks), generator=gen).repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)
    a = _quantized(torch.ldexp(randn(1, m, k), ea).float(), 1)
    b = _quantized(torch.ldexp(randn(2, n, k), eb).float(), 128)
    _check(a, b, k, out)
