"""jenga_rms_norm and its gradient against float64, through the binding.  Tolerances: more_operator_util."""
import math

import pytest
import torch

from more_operator_util import quantize_mx, rms, rms_grad, values_mx
from operator_util import TYPES, U32, check, half_step, held_values, quantize, randn

pytestmark = pytest.mark.gpu
EPS = 1e-6
PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]


def _inputs(rows, cols, dtype, params, seed, heads=None):
    shape = (rows, cols) if heads is None else (rows, heads, cols)
    x = (randn(seed, *shape) * (0.5 + randn(seed + 1, cols).abs()) + 0.7 * randn(seed + 2, cols)).to(TYPES[dtype])
    return x, (1 + 0.4 * randn(seed + 3, cols)).to(TYPES[params]), randn(seed + 4, *shape).to(TYPES[dtype])


def _tol(want, slack, dtype):
    return half_step(dtype) * want.abs() + slack * (1 + half_step(dtype)) + (2.0 ** -25 if dtype == torch.float16 else 0)


SIZES = [(1, 1), (2, 3), (5, 8), (7, 64), (33, 65), (9, 128), (70, 129), (3, 256), (5, 300), (6, 512), (5, 513), (4, 1000), (3, 1024), (7, 1025),
         (11, 1536), (2, 1537), (3, 2048), (2, 3001), (3, 4096), (2, 5120), (2, 6145), (2, 8192), (3, 9999), (1, 12288), (2, 12289), (2, 16384),
         (2, 16385), (1, 131072), (3000, 72)]


@pytest.mark.parametrize("dtype,params", PAIRS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_gradient(rows, cols, dtype, params):
    import paper_2505_16864_amd as J
    x, w, add = _inputs(rows, cols, dtype, params, 3 * rows + cols)
    t = x.dtype
    total = (x.float() + add.float()).to(t)
    want, slack, r = rms(total.double(), w.double(), 0.25, EPS)
    y, s, rstd = torch.full_like(x, 7, device="cuda:0"), torch.full_like(x, 7, device="cuda:0"), torch.full((rows,), 7.0, device="cuda:0")
    J.jenga_rms_norm(x.cuda(), y, w.cuda(), residual=add.cuda(), total=s, rstd=rstd, weight_offset=0.25, eps=EPS)
    assert torch.equal(s.cpu(), total)
    check(y, want, _tol(want, slack, t), "y")
    check(rstd, r, 90 * U32 * r, "rstd")
    # the norm alone, and the gradient from it
    want, slack, _ = rms(x.double(), w.double(), 0.0, EPS)
    J.jenga_rms_norm(x.cuda(), y, w.cuda(), rstd=rstd, eps=EPS)
    check(y, want, _tol(want, slack, t), "y alone")
    dy, dt = randn(rows + 1, rows, cols).to(t), randn(rows + 2, rows, cols).to(t)
    for more in (None, dt):
        dx, dw = torch.full_like(x, 7, device="cuda:0"), torch.full((cols,), 7.0, device="cuda:0")
        room = torch.empty(J.jenga_rms_norm_grad_workspace(rows, cols), dtype=torch.uint8, device="cuda:0")
        J.jenga_rms_norm_grad(x.cuda(), dy.cuda(), dx, w.cuda(), rstd, dtotal=None if more is None else more.cuda(), dweight=dw, workspace=room)
        wx, sx, ww, sw = rms_grad(x.double(), dy.double(), w.double(), 0.0, rstd.cpu().double(), torch.zeros(()) if more is None else more.double())
        check(dx, wx, _tol(wx, sx, t), "dx")
        check(dw, ww, sw, "dweight")
        again = torch.full_like(dx, 3)
        J.jenga_rms_norm_grad(x.cuda(), dy.cuda(), again, w.cuda(), rstd, dtotal=None if more is None else more.cuda())
        assert torch.equal(again, dx)


# Heads of a projection's columns: Q and K where one product left them, each row of each head by itself, one weight.
@pytest.mark.parametrize("rows,heads,cols", [(1, 2, 64), (37, 5, 72), (300, 3, 128), (20, 40, 96), (9, 12, 100), (4, 7, 520), (3, 2, 3000), (2, 3, 17000)])
@pytest.mark.parametrize("dtype,params", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_heads(rows, heads, cols, dtype, params):
    import paper_2505_16864_amd as J
    x, w, _ = _inputs(rows, cols, dtype, params, cols + heads, 3 * heads)
    qkv = x.cuda().view(rows, 3, heads, cols)
    for i, in_place in ((0, False), (1, False), (1, True)):
        mine = x.view(rows, 3, heads, cols)[:, i]
        want, slack, r = rms(mine.double(), w.double(), 0.0, EPS)
        y = qkv[:, i] if in_place else torch.empty((rows, heads, cols), dtype=x.dtype, device="cuda:0")
        rstd = torch.empty((rows, heads), device="cuda:0")
        before = qkv.clone()
        J.jenga_rms_norm(qkv[:, i], y, w.cuda(), rstd=rstd, eps=EPS)
        check(y, want, _tol(want, slack, x.dtype), "head %d" % i)
        check(rstd, r, 90 * U32 * r, "rstd")
        for other in range(3):
            if not (in_place and other == i):
                assert torch.equal(qkv[:, other], before[:, other])
    mine = x.view(rows, 3, heads, cols)[:, 0]
    _, _, r = rms(mine.double(), w.double(), 0.0, EPS)
    rstd = r.float().cuda()
    dy = randn(5, rows, heads, cols).to(x.dtype)
    grads, dw = torch.zeros((rows, 3, heads, cols), dtype=x.dtype, device="cuda:0"), torch.empty(cols, device="cuda:0")
    room = torch.empty(J.jenga_rms_norm_grad_workspace(rows * heads, cols), dtype=torch.uint8, device="cuda:0")
    J.jenga_rms_norm_grad(qkv[:, 0], dy.cuda(), grads[:, 1], w.cuda(), rstd, dweight=dw, workspace=room)
    wx, sx, ww, sw = rms_grad(mine.double(), dy.double(), w.double(), 0.0, rstd.cpu().double(), torch.zeros(()))
    check(grads[:, 1], wx, _tol(wx, sx, x.dtype), "dx")
    check(dw, ww, sw, "dweight")
    assert not grads[:, 0].any() and not grads[:, 2].any()


# Rows that lie apart and off the 16-byte grid, a residual stream updated in place, a gradient that is the same for all rows.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [96, 777, 5121, 20001])
def test_strides_and_in_place(cols, dtype):
    import paper_2505_16864_amd as J
    rows = 6
    x, w, add = _inputs(rows, cols, dtype, dtype, cols)
    total = (x.float() + add.float()).to(x.dtype)
    want, slack, _ = rms(total.double(), w.double(), 0.0, EPS)
    room = torch.full((rows, 2 * cols + 5), 3.0, dtype=x.dtype, device="cuda:0")
    room[:, 1:1 + cols], room[:, cols + 3:2 * cols + 3] = x.cuda(), add.cuda()
    xs, stream = room[:, 1:1 + cols], room[:, cols + 3:2 * cols + 3]
    y = torch.empty((rows, cols + 7), dtype=x.dtype, device="cuda:0")[:, 3:3 + cols]
    J.jenga_rms_norm(xs, y, w.cuda(), residual=stream, total=stream, eps=EPS)
    check(y, want, _tol(want, slack, x.dtype), "y")
    assert torch.equal(stream.cpu(), total) and torch.equal(xs.cpu(), x)
    assert all(bool((room[:, a:b] == 3).all()) for a, b in ((0, 1), (cols + 1, cols + 3), (2 * cols + 3, 2 * cols + 5)))
    J.jenga_rms_norm(xs, xs, w.cuda(), residual=add.cuda(), total=None, eps=EPS)        # over x, nothing else kept
    check(xs, want, _tol(want, slack, x.dtype), "over x")
    rstd = torch.rand(rows, device="cuda:0") + 0.5
    dy = randn(3, cols).to(x.dtype)
    into = randn(4, rows, cols).to(x.dtype)
    dx = into.cuda()
    J.jenga_rms_norm_grad(stream, dy.cuda().expand(rows, cols), dx, None, rstd, dtotal=dx, weight_offset=1.0)
    wx, sx, _, _ = rms_grad(total.double(), dy.double().expand(rows, cols), torch.zeros(cols, dtype=torch.float64), 1.0, rstd.cpu().double(), into.double())
    check(dx, wx, _tol(wx, sx, x.dtype), "dx over dtotal")


# Zero rows, rows of one value, large and small ones, infinities and NaN: the others keep their values.
@pytest.mark.parametrize("cols", [96, 777, 9000, 20000])
def test_rows_that_are_not_ordinary(cols):
    import paper_2505_16864_amd as J
    x = randn(5, 7, cols).float()
    x[0], x[1] = 0, 2.5
    x[2] *= 1e15
    x[3] *= 1e-12
    x[4, cols // 2] = float("inf")
    x[5, cols - 1] = float("nan")
    y, rstd = torch.empty(7, cols, device="cuda:0"), torch.empty(7, device="cuda:0")
    J.jenga_rms_norm(x.cuda(), y, None, rstd=rstd, eps=0.0, weight_offset=1.0)
    want, slack, _ = rms(x.double(), torch.zeros(cols, dtype=torch.float64), 1.0, 0.0)
    got = y.cpu()
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isnan(got[5]).all()) and bool(torch.isnan(got[4, cols // 2]))   # 0 / 0 with no eps
    for i in (1, 2, 3, 6):
        check(got[i], want[i], U32 * want[i].abs() + slack[i] + 2.0 ** -149, "row %d" % i)
    dx, dw = torch.empty(7, cols, device="cuda:0"), torch.empty(cols, device="cuda:0")
    rstd[0] = math.inf                                            # as a row of zeros leaves it
    room = torch.empty(J.jenga_rms_norm_grad_workspace(7, cols), dtype=torch.uint8, device="cuda:0")
    dy = randn(6, 7, cols).float()
    J.jenga_rms_norm_grad(x.cuda(), dy.cuda(), dx, None, rstd, dweight=dw, workspace=room, weight_offset=1.0)
    wx, sx, _, _ = rms_grad(x.double(), dy.double(), torch.zeros(cols, dtype=torch.float64), 1.0, rstd.cpu().double(), torch.zeros(()))
    for i in (1, 3, 6):
        check(dx.cpu()[i], wx[i], _tol(wx, sx, torch.float32)[i] + 2.0 ** -149, "dx %d" % i)


# The gradient's formula is the derivative: differences of the plain form, on the CPU.
def test_formula_against_differences():
    cols, w0 = 13, 0.3
    x, w, dy = randn(1, 4, cols), randn(2, cols), randn(3, 4, cols)
    loss = lambda a, b: (rms(a, b, w0, EPS)[0] * dy).sum()  # noqa: E731
    dx, _, dw, _ = rms_grad(x, dy, w, w0, rms(x, w, w0, EPS)[2], torch.zeros(()))
    step = 1e-5
    for i in range(cols):
        e = torch.zeros(cols, dtype=torch.float64)
        e[i] = step
        for r in range(4):
            d = torch.zeros_like(x)
            d[r, i] = step
            assert abs((loss(x + d, w) - loss(x - d, w)) / (2 * step) - dx[r, i]) < 1e-7
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - dw[i]) < 1e-7


# Results straight to 8 and 4 bits: those of the norm in float32, quantised.  A float32 result off by the slack may fall on the other side of a
# border between two values, and the largest of a block on the other side of a border between two scales: then the value is the neighbour's, a whole
# step instead of half of one, and the step twice as large.
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 100), (5, 128), (4, 130), (7, 513), (3, 1001), (33, 1536), (2, 3001), (2, 5120), (2, 8200), (2, 14000), (1, 20001)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_results_of_few_bits(rows, cols, dtype):
    import paper_2505_16864_amd as J
    x, w, add = _inputs(rows, cols, dtype, dtype, 31 + cols)
    total = (x.float() + add.float()).to(x.dtype)
    want, slack, _ = rms(total.double(), w.double(), 0.0, EPS)
    padded = J.padded_columns(cols)
    s = torch.empty_like(x, device="cuda:0")
    for bits in (8, 4):
        if bits == 8:
            q = torch.full((rows, padded), 77, dtype=torch.uint8, device="cuda:0").view(torch.float8_e4m3fn)
            scale = torch.full((rows, J.scale_columns(cols)), 77, dtype=torch.uint8, device="cuda:0")
        else:
            q = torch.full((rows, padded // 2), 77, dtype=torch.uint8, device="cuda:0")
            scale = torch.full((rows, padded // 32), 77, dtype=torch.uint8, device="cuda:0")
        J.jenga_rms_norm(x.cuda(), q, w.cuda(), residual=add.cuda(), total=s, y_scale=scale, eps=EPS)
        assert torch.equal(s.cpu(), total)
        if bits == 8:
            held, bytes_ = quantize(want, 1)
            got, step = held_values(q, scale, 1), 2.0 ** -3
        else:
            codes, bytes_ = quantize_mx(want)
            held, got, step = values_mx(codes, bytes_), values_mx(q, scale), 1.0
        off = (scale.cpu().int() - bytes_.int()).abs()
        assert int(off.max()) <= 1 and float((off > 0).double().mean()) <= 0.02 + 1.5 / off.numel()
        differ = got != held
        assert float(differ.double().mean()) <= 0.005 + 1.5 / differ.numel()
        full = torch.zeros_like(got)
        full[:, :cols] = want.abs()
        unit = torch.ldexp(torch.ones(bytes_.shape, dtype=torch.float64), bytes_.int() - 127).repeat_interleave(128 if bits == 8 else 32, 1)[:, :padded]
        assert bool(((got - held).abs() <= 2 * step * torch.maximum(full, unit * (2.0 ** -6 if bits == 8 else 1.0))).all())
        assert not got[:, cols:].any()


# A block with an infinity is all NaN in 4 bits, and its value NaN in 8 bits; blocks beside it are what they were.
def test_few_bits_of_what_is_not_finite():
    import paper_2505_16864_amd as J
    w = torch.ones(256)
    w[40] = float("inf")
    x = randn(1, 3, 256).float()
    q, s = torch.empty((3, 128), dtype=torch.uint8, device="cuda:0"), torch.empty((3, 8), dtype=torch.uint8, device="cuda:0")
    J.jenga_rms_norm(x.cuda(), q, w.cuda(), y_scale=s, eps=EPS)
    got = values_mx(q, s)
    assert bool(torch.isnan(got[:, 32:64]).all()) and not torch.isnan(got[:, :32]).any() and not torch.isnan(got[:, 64:]).any()


# Rows past 2^31 elements of a tensor, and more rows with heads than a grid takes at once.
def test_far_rows():
    import paper_2505_16864_amd as J
    rows, cols = 300000, 128
    wide = torch.zeros((rows, 7200 * 2), dtype=torch.bfloat16, device="cuda:0")[:, 14208:14336]
    x = randn(8, 1000, cols).to(torch.bfloat16)
    wide[-1000:] = x.cuda()
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda:0")
    J.jenga_rms_norm(wide, y, None, weight_offset=1.0, eps=EPS)
    want, slack, _ = rms(x.double(), torch.zeros(cols, dtype=torch.float64), 1.0, EPS)
    check(y[-1000:], want, _tol(want, slack, torch.bfloat16), "far")
    assert not y[:-1000].any()
