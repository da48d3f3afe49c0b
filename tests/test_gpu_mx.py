"""jenga_quantize_mx and jenga_matmul_mx against float64, through the binding.

Tolerances.  Products of two values and their scales are exact; of k of them added in float32, in any order, the sum is off by at most
k u times the sum of their magnitudes (u = 2^-24), and is rounded once to the result's type behind the addition of the bias, which is one more u."""
import pytest
import torch

from more_operator_util import quantize_mx, values_mx
from operator_util import TYPES, U32, check, half_step, randn

pytestmark = pytest.mark.gpu


def _empty(rows, cols):
    import paper_2505_16864_amd as J
    padded = J.padded_columns(cols)
    return [torch.full((rows, padded // n), 77, dtype=torch.uint8, device="cuda:0") for n in (2, 32)]


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (2, 127), (5, 128), (7, 500), (4, 512), (3, 513), (65, 1000), (2, 5120), (2, 131072), (3000, 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_quantize(rows, cols, dtype):
    import paper_2505_16864_amd as J
    x = (randn(cols, rows, cols) * torch.exp2(3 * randn(cols + 1, rows, cols))).to(TYPES[dtype])
    wide = torch.full((rows, cols + 5), float("nan"), dtype=x.dtype, device="cuda:0")
    wide[:, 3:3 + cols] = x.cuda()
    q, scale = _empty(rows, cols)
    J.jenga_quantize_mx(wide[:, 3:3 + cols], q, scale)
    want, want_scale = quantize_mx(x.double())
    assert torch.equal(scale.cpu(), want_scale) and torch.equal(q.cpu(), want)


# Every border between two values and its neighbours, blocks of zeros, the largest and smallest numbers, infinities and NaN.
def test_quantize_borders():
    import paper_2505_16864_amd as J
    marks = torch.tensor([0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0])
    near = torch.cat([marks, torch.nextafter(marks, torch.tensor(0.0)), torch.nextafter(marks, torch.tensor(9.0)).clamp(max=6.0)])
    x = torch.zeros((60, 128))
    for row, e in enumerate(list(range(-126, 124, 6))[:42]):
        x[row, :42] = near * 2.0 ** e
        x[row, 31], x[row, 32] = 6.0 * 2.0 ** e, -6.0 * 2.0 ** e
        x[row, 42:64] = -near[:22] * 2.0 ** e
    x[43, 5] = torch.finfo(torch.float32).max
    x[44, 5], x[44, 40] = 2.0 ** -149, -2.0 ** -126
    x[45, 0], x[45, 33], x[45, 64] = float("inf"), float("nan"), -float("inf")
    x[46, :32] = -0.0
    x[47, 3], x[47, 40] = torch.nextafter(torch.tensor(6.0), torch.tensor(9.0)), 12.0
    q, scale = _empty(60, 128)
    J.jenga_quantize_mx(x.cuda(), q, scale)
    want, want_scale = quantize_mx(x.double())
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(q.cpu(), want)


SIZES = [(1, 128, 1), (1, 384, 17), (3, 256, 64), (16, 1536, 100), (17, 512, 33), (32, 640, 300), (33, 128, 64), (65, 384, 200), (130, 1024, 129),
         (300, 256, 1000), (777, 1024, 1111), (64, 5120, 8192), (1, 5120, 640), (513, 896, 4500), (2100, 640, 2050), (1040, 384, 16400)]


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_product(m, k, n, out):
    import paper_2505_16864_amd as J
    gen = torch.Generator().manual_seed(m + k + n)
    operands = []
    for rows in (m, n):      # all codes; scales over many powers of two, as a row's largest values make them
        q = torch.randint(0, 256, (rows, k // 2), generator=gen, dtype=torch.uint8)
        s = torch.randint(118, 131, (rows, k // 32), generator=gen, dtype=torch.uint8)
        operands += [q, s]
    bias = randn(5, n).float() if n % 2 else None
    a, b = values_mx(*operands[:2]), values_mx(*operands[2:])
    want, mags = a @ b.t(), a.abs() @ b.abs().t()
    if bias is not None:
        want = want + bias.double()
        mags = mags + bias.double().abs()
    room = torch.full((m, n + 3), 5.0, dtype=TYPES[out], device="cuda:0")
    got = room[:, :n]
    J.jenga_matmul_mx(operands[0].cuda(), operands[1].cuda(), operands[2].cuda(), operands[3].cuda(), got, None if bias is None else bias.cuda())
    slack = (k + 2) * U32 * mags
    check(got, want, half_step(got.dtype) * (want.abs() + slack) + slack + (2.0 ** -25 if out == "f16" else 0))
    assert bool((room[:, n:] == 5).all())


# Sums whose parts have scales far apart, as neighbouring blocks of 32 columns do: small ones are not lost beside large ones that cancel.
@pytest.mark.parametrize("m,n", [(1, 40), (40, 40), (600, 1300)])
def test_product_of_distant_scales(m, n):
    import paper_2505_16864_amd as J
    k, gen = 512, torch.Generator().manual_seed(3)
    q, w = [torch.randint(0, 256, (r, k // 2), generator=gen, dtype=torch.uint8) for r in (m, n)]
    s, t = [torch.full((r, k // 32), 127, dtype=torch.uint8) for r in (m, n)]
    s[:, ::2] = 127 - 18
    # the large blocks: the second half of their columns takes off what the first adds
    for block in range(1, k // 32, 2):
        at = block * 16
        q[:, at + 8:at + 16], w[:, at + 8:at + 16] = q[:, at:at + 8] ^ 0x88, w[:, at:at + 8]
    a, b = values_mx(q, s), values_mx(w, t)
    want, mags = a @ b.t(), a.abs() @ b.abs().t()
    got = torch.empty((m, n), device="cuda:0")
    J.jenga_matmul_mx(q.cuda(), s.cuda(), w.cuda(), t.cuda(), got)
    check(got, want, k * U32 * mags)


# A scale of 255 makes NaN of every result that it is part of, and of no other; extreme scales; rows and columns past the ends of the operands are not looked at.
@pytest.mark.parametrize("m,n", [(5, 40), (70, 130), (600, 1300)])
def test_scales_at_the_ends(m, n):
    import paper_2505_16864_amd as J
    k, gen = 384, torch.Generator().manual_seed(m)
    q, w = [torch.randint(0, 256, (r, k // 2), generator=gen, dtype=torch.uint8) for r in (m, n)]
    s, t = [torch.full((r, k // 32), 127, dtype=torch.uint8) for r in (m, n)]
    s[2, 11], t[7, 0] = 255, 255
    s[3], t[:6] = 0, 230                   # 2^-127 times 2^103
    s[4], t[8:12] = 240, 20                # 2^113 times 2^-107
    a, b = values_mx(q, s), values_mx(w, t)
    want, mags = a @ b.t(), a.abs() @ b.abs().t()
    want[2], want[:, 7] = float("nan"), float("nan")
    got = torch.empty((m, n), device="cuda:0")
    J.jenga_matmul_mx(q.cuda(), s.cuda(), w.cuda(), t.cuda(), got)
    # 2^113 times 2^103 times 0.25 or more is past float32's 2^128: what becomes of sums of such products, of both signs, is not said
    got[4, :6], want[4, :6] = 0, 0
    # sums below 2^-126 may be taken as 0
    check(got, want, k * U32 * torch.nan_to_num(mags) + 2.0 ** -126)


def test_quantized_norm_times_weight_in_a_graph():
    import paper_2505_16864_amd as J
    rows, cols, n = 300, 1000, 700
    x = randn(1, rows, cols).to(torch.bfloat16).cuda()
    w = (randn(2, n, cols) / 30).to(torch.bfloat16).cuda()
    (a, s), (b, t) = _empty(rows, cols), _empty(n, cols)
    out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda:0")
    J.jenga_quantize_mx(w, b, t)

    def run():
        J.jenga_rms_norm(x, a, None, y_scale=s, weight_offset=1.0)
        J.jenga_matmul_mx(a, s, b, t, out)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.copy_(randn(10 + i, rows, cols).to(torch.bfloat16))
        graph.replay()
        got = out.clone()
        out.zero_()
        run()
        assert torch.equal(got, out)
