"""jenga_quantize and jenga_matmul against float64, through the C ABI.

Tolerances.  Quantisation is exact: powers of two, one rounding.  Products for 16-bit results: the f8 matrix core adds eight products at
a time, each cut off at 2^-13 of the largest of the eight, so a result is off by at most 8 * 2^-13 of the sum of the products'
magnitudes; the float32 sums behind it are below that.  Over many results those errors have no common sign: their root mean square
is held to 2^-12 of the results', beside the rounding's 2^-9 (bf16) or 2^-12 (fp16).  Float32 results: k float32 additions in some order,
k 2^-24 of the sum of magnitudes, and 2^-19 in the root mean square."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, held_values, quantize, randn

pytestmark = pytest.mark.gpu


def _quantized(x, block_rows):
    import paper_2505_16864_amd as J
    rows, cols = x.shape
    q = torch.full((rows, J.padded_columns(cols)), 0x55, dtype=torch.uint8, device="cuda:0").view(torch.float8_e4m3fn)
    scale = torch.full((-(-rows // block_rows), J.scale_columns(cols)), 99, dtype=torch.uint8, device="cuda:0")
    J.jenga_quantize(x, q, scale, block_rows)
    return q, scale


def _same(got, want):
    return bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 127), (5, 129), (128, 512), (129, 513), (260, 1000), (2, 9000)])
def test_quantize(rows, cols, block_rows, dtype):
    x = (randn(rows + cols, rows, cols) * torch.exp(3 * randn(7, cols))).to(TYPES[dtype])
    q, scale = _quantized(x.cuda(), block_rows)
    torch.cuda.synchronize()
    want, want_scale = quantize(x.double(), block_rows)
    assert torch.equal(scale.cpu(), want_scale)
    assert _same(held_values(q, scale, block_rows), want)


# Every border between two e4m3 values, blocks of zeros, the smallest and largest magnitudes, borders between two scales, infinities
# and NaN, which count for no scale.
def test_quantize_at_the_borders():
    values = []
    for e in range(-9, 9):
        for m in range(16, 33):
            values.append(m / 16.0 * 2.0 ** e)                       # values and the middles between them
    v = torch.tensor(values, dtype=torch.float64)
    rows = [torch.cat([v, -v, torch.tensor([448.0] * 4, dtype=torch.float64)])]
    rows.append(torch.nextafter(rows[0].float(), torch.tensor(1e30)).double())
    rows.append(torch.nextafter(rows[0].float(), torch.tensor(-1e30)).double())
    n = rows[0].numel()
    pad = -(-n // 128) * 128 - n
    x = torch.cat([torch.nn.functional.pad(r, (0, pad), value=448.0).view(-1, 128) for r in rows])
    more = torch.zeros((12, 128), dtype=torch.float64)
    more[1, 5] = 448.0 * 2.0 ** -20
    more[2, 5] = float(torch.nextafter(torch.tensor(448.0 * 2.0 ** -20), torch.tensor(1.0)))
    more[3, 5], more[3, 6] = 3.0e38, -1.0
    more[4, 5] = 2.0 ** -126
    more[5, 5] = 2.0 ** -149                                         # the smallest float32
    more[6, 3], more[6, 4], more[6, 5] = float("inf"), float("-inf"), 3.0
    more[7, 3], more[7, 5] = float("nan"), -5.0
    more[8, :] = float("nan")
    more[9, 0], more[9, 1] = 448.0, 2.0 ** -9
    more[10, 0], more[10, 1] = 448.0, -0.0
    more[11, :] = 480.0
    x = torch.cat([x, more]).float()
    q, scale = _quantized(x.cuda(), 1)
    torch.cuda.synchronize()
    want, want_scale = quantize(x.double(), 1)
    assert torch.equal(scale.cpu(), want_scale)
    assert _same(held_values(q, scale, 1), want)
    q, scale = _quantized(x.cuda(), 128)
    want, want_scale = quantize(x.double(), 128)
    assert torch.equal(scale.cpu(), want_scale) and _same(held_values(q, scale, 128), want)


def test_quantize_rows_that_lie_apart():
    x = randn(3, 37, 300).to(torch.bfloat16)
    room = torch.full((37, 701), 1000.0, dtype=torch.bfloat16, device="cuda:0")
    room[:, 3:303] = x.cuda()
    for block_rows in (1, 128):
        q, scale = _quantized(room[:, 3:303], block_rows)
        want, want_scale = quantize(x.double(), block_rows)
        assert torch.equal(scale.cpu(), want_scale) and _same(held_values(q, scale, block_rows), want)


def _product(m, n, k, out, bias, seed, tails=False):
    import paper_2505_16864_amd as J
    x, w = randn(seed, m, k), randn(seed + 1, n, k) * torch.exp(randn(seed + 3, n, 1))
    if tails:
        x, w = x ** 3, w ** 3
    a, a_scale = _quantized(x.float().cuda(), 1)
    b, b_scale = _quantized(w.float().cuda(), 128)
    bias = randn(seed + 2, n).float() if bias else None
    got = torch.full((m, n), 7.0, dtype=TYPES[out], device="cuda:0")
    J.jenga_matmul(a, a_scale, b, b_scale, got, bias.cuda() if bias is not None else None)
    torch.cuda.synchronize()
    A, B = held_values(a, a_scale, 1), held_values(b, b_scale, 128)
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    return got, want, size


def _check_product(got, want, size, k, out, what):
    dtype = TYPES[out]
    rms = lambda t: float(t.square().mean().sqrt())  # noqa: E731
    err = rms(got.cpu().double() - want) / rms(want)
    if out == "f32":
        check(got, want, U32 * (k + 8) * size, what)
        assert err <= 2.0 ** -19, (what, err)
    else:
        check(got, want, half_step(dtype) * want.abs() * 1.01 + 8 * 2.0 ** -13 * size, what)
        assert err <= {"bf16": 2.0 ** -9, "f16": 2.0 ** -12}[out] + 2.0 ** -12, (what, err)


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 128), (1, 1000, 640), (2, 129, 1536), (5, 300, 1000), (16, 512, 2048),
                                   (17, 48, 256), (31, 4096, 384), (33, 640, 512), (64, 257, 1280), (65, 128, 128), (100, 1111, 777),
                                   (128, 256, 512), (129, 385, 130), (200, 200, 5120), (257, 512, 1024), (300, 260, 640),
                                   (513, 1025, 384), (1000, 768, 896)])
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
def test_product(m, n, k, out):
    got, want, size = _product(m, n, k, out, (m + n) % 2 == 0, m + n + k)
    _check_product(got, want, size, k, out, "%d x %d x %d" % (m, n, k))


@pytest.mark.parametrize("m,n,k", [(1, 256, 1024), (40, 300, 640), (300, 300, 640)])
def test_float32_products_of_long_tails_lose_nothing(m, n, k):
    got, want, size = _product(m, n, k, "f32", False, 17, tails=True)
    _check_product(got, want, size, k, "f32", "long tails")


# Many tiles in both directions, many steps: every result against a float64 product on the GPU.
@pytest.mark.parametrize("m,n,k,out", [(2500, 3000, 2048, "bf16"), (1300, 2900, 640, "f16"), (700, 9000, 512, "bf16"),
                                       (9000, 700, 1152, "f32"), (4500, 5200, 256, "bf16")])
def test_larger_products(m, n, k, out):
    import paper_2505_16864_amd as J
    gen = torch.Generator(device="cuda:0").manual_seed(m)
    x = torch.randn((m, k), generator=gen, device="cuda:0")
    w = torch.randn((n, k), generator=gen, device="cuda:0")
    a, a_scale = _quantized(x, 1)
    b, b_scale = _quantized(w, 128)
    got = torch.full((m, n), 7.0, dtype=TYPES[out], device="cuda:0")
    J.jenga_matmul(a, a_scale, b, b_scale, got)
    A, B = held_values(a, a_scale, 1).cuda(), held_values(b, b_scale, 128).cuda()
    want, size = (A @ B.t()).cpu(), (A.abs() @ B.abs().t()).cpu()
    _check_product(got, want, size, k, out, "larger")


def test_rows_of_the_result_lie_apart_and_nothing_else_is_written():
    import paper_2505_16864_amd as J
    for m, n, k, out in ((3, 70, 256, "bf16"), (150, 200, 384, "bf16"), (300, 300, 256, "f32"), (270, 515, 128, "f16")):
        a, a_scale = _quantized(randn(1, m, k).float().cuda(), 1)
        b, b_scale = _quantized(randn(2, n, k).float().cuda(), 128)
        alone = torch.empty((m, n), dtype=TYPES[out], device="cuda:0")
        J.jenga_matmul(a, a_scale, b, b_scale, alone)
        room = torch.full((m + 2, n + 13), 5.0, dtype=TYPES[out], device="cuda:0")
        J.jenga_matmul(a, a_scale, b, b_scale, room[1:m + 1, 3:3 + n])
        torch.cuda.synchronize()
        assert torch.equal(room[1:m + 1, 3:3 + n], alone)
        room[1:m + 1, 3:3 + n] = 5.0
        assert bool((room == 5.0).all())


# Infinities and NaN of an activation make its row NaN, and no other.
def test_a_row_that_is_not_finite_stays_alone():
    import paper_2505_16864_amd as J
    for m in (4, 200):
        for out in ("bf16", "f32"):
            x = randn(3, m, 256).float()
            x[1, 200], x[3, 5] = float("nan"), float("inf")
            a, a_scale = _quantized(x.cuda(), 1)
            b, b_scale = _quantized(randn(4, 100, 256).float().cuda(), 128)
            got = torch.empty((m, 100), dtype=TYPES[out], device="cuda:0")
            J.jenga_matmul(a, a_scale, b, b_scale, got)
            bad = torch.isnan(got.cpu())
            assert bool(bad[1].all()) and bool(bad[3].all()) and int(bad.sum()) == 200


# The gradients by the same call: da = dout b, from b's transpose; db = dout^T a, from the transposes of both.
@pytest.mark.parametrize("m,n,k", [(70, 200, 300), (260, 384, 256)])
def test_gradients_are_products_of_the_same_kind(m, n, k):
    import paper_2505_16864_amd as J
    x, w, dout = [randn(s, *shape).float() for s, shape in ((1, (m, k)), (2, (n, k)), (3, (m, n)))]
    for left, right in ((dout, w.t()), (dout.t(), x.t())):
        a, a_scale = _quantized(left.contiguous().cuda(), 1)
        b, b_scale = _quantized(right.contiguous().cuda(), 128)
        got = torch.empty((left.shape[0], right.shape[0]), device="cuda:0")
        J.jenga_matmul(a, a_scale, b, b_scale, got)
        torch.cuda.synchronize()
        A, B = quantize(left.double(), 1)[0], quantize(right.double(), 128)[0]
        check(got, A @ B.t(), U32 * (A.shape[1] + 8) * (A.abs() @ B.abs().t()), "gradient")
        full = left.double() @ right.double().t()
        # each value of either operand is off by at most 2^-4 of itself, or 2^-10 of its block's unit: about 3 % of the norm
        assert float((got.cpu().double() - full).norm() / full.norm()) <= 2 * 2.0 ** -4
    # the transpose of a matrix in blocks of 128 x 128 holds the same values
    held, turned = quantize(w.double(), 128)[0][:, :k], quantize(w.double().t(), 128)[0][:, :n]
    assert torch.equal(held, turned.t())
