"""Layer norm's gradient where mean and 1 / spread are so far apart that (0 - mean) * rstd is no float32: values that are not there (columns
behind a row's last one, rows behind the last one) have to stay out of every sum.

A row whose values are all 2^120 has mean 2^120 exactly (up to 255 of them add up below 2^128, a power of two times a whole number), no
spread, h = 0 and rstd = 1 / sqrt(eps) = 2^10 for eps = 2^-20.  So dx = rstd (g - mean(g)), dweight = 0 and dbias = the sum of dy."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, held_values, quantize, randn

pytestmark = pytest.mark.gpu


# One row and several; columns that fill no piece of a row, and less than eight columns.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 3), (1, 8), (5, 100), (7, 104), (3, 250), (9, 255)])
def test_constant_rows_far_off_zero(rows, cols, dtype):
    import paper_2505_16864_amd as J
    x = torch.full((rows, cols), 2.0 ** 120, dtype=TYPES[dtype])
    w = randn(1, cols).float()
    dy = randn(2, rows, cols).to(x.dtype)
    gx, mean, rstd = x.cuda(), torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
    y, dx = torch.empty_like(gx), torch.empty_like(gx)
    J.jenga_layer_norm(gx, y, w.cuda(), mean=mean, rstd=rstd, eps=2.0 ** -20)
    dw, db = torch.empty(cols, device="cuda:0"), torch.empty(cols, device="cuda:0")
    ws = torch.empty(J.jenga_layer_norm_grad_workspace(rows, cols), dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm_grad(gx, dy.cuda(), dx, w.cuda(), mean, rstd, dw, db, ws)
    torch.cuda.synchronize()
    assert bool((mean == 2.0 ** 120).all()) and not y.any()
    check(rstd, torch.full((rows,), 2.0 ** 10, dtype=torch.float64), torch.tensor(4 * U32 * 2.0 ** 10, dtype=torch.float64), "rstd")
    g = dy.double() * w.double()
    want = 2.0 ** 10 * (g - g.mean(1, keepdim=True))
    # at most 140 additions follow each other for the mean, a handful of roundings besides
    slack = U32 * 2.0 ** 10 * (8 * g.abs() + 150 * g.abs().mean(1, keepdim=True))
    check(dx, want, half_step(x.dtype) * want.abs() + slack * 1.01, "dx")
    assert not dw.any()
    check(db, dy.double().sum(0), U32 * (rows + 8) * dy.double().abs().sum(0), "dbias")


# The same through every kernel by statistics that the caller hands in: mean 2^100 = x, rstd 2^30, so that h is 0 where a value is and
# 2^130 in magnitude, an infinity, where none is.
@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("cols", [3, 100, 777, 1000, 1500, 2000, 2500, 5000, 8000, 8191, 8200, 9001])
def test_statistics_far_apart(rows, cols):
    import paper_2505_16864_amd as J
    x = torch.full((rows, cols), 2.0 ** 100, device="cuda:0")
    mean, rstd = torch.full((rows,), 2.0 ** 100, device="cuda:0"), torch.full((rows,), 2.0 ** 30, device="cuda:0")
    dy = randn(3, rows, cols).float()
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda:0"), torch.empty(cols, device="cuda:0")
    ws = torch.empty(J.jenga_layer_norm_grad_workspace(rows, cols), dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm_grad(x, dy.cuda(), dx, None, mean, rstd, dw, db, ws, weight_offset=1.0)
    torch.cuda.synchronize()
    g = dy.double()
    want = 2.0 ** 30 * (g - g.mean(1, keepdim=True))
    slack = U32 * 2.0 ** 30 * (8 * g.abs() + 150 * g.abs().mean(1, keepdim=True))
    check(dx, want, half_step(torch.float32) * want.abs() + slack * 1.01, "dx")
    assert not dw.any()
    check(db, g.sum(0), U32 * (rows + 8) * g.abs().sum(0), "dbias")


# 8-bit results with a scale and a shift for each of several groups, one of them short, rows that lie apart, an odd number of columns too:
# the bits that quantising the float32 result gives, but where that is a rounding's width off a border.
@pytest.mark.parametrize("rows,cols,group_rows", [(10, 96, 4), (7, 1000, 1), (33, 1536, 12), (5, 130, 2), (9, 2048, 5), (3, 8200, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_eight_bit_results_of_groups(rows, cols, group_rows, dtype):
    import paper_2505_16864_amd as J
    groups = -(-rows // group_rows)
    room = randn(rows + cols, rows, cols + 7).to(TYPES[dtype]).cuda()
    x = room[:, 3:3 + cols]
    params = (0.4 * randn(3, groups, 2 * cols + 1)).to(TYPES[dtype]).cuda()
    w, b = params[:, :cols], params[:, cols + 1:]
    q = torch.full((rows, J.padded_columns(cols)), 99, dtype=torch.uint8, device="cuda:0")
    s = torch.full((rows, J.scale_columns(cols)), 99, dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm(x, q, w, b, y_scale=s, group_rows=group_rows, weight_offset=1.0)
    y = torch.empty((rows, cols), device="cuda:0")
    J.jenga_layer_norm(x.float(), y, w.float(), b.float(), group_rows=group_rows, weight_offset=1.0)
    torch.cuda.synchronize()
    want, want_scale = quantize(y.cpu().double(), 1)
    got = held_values(q, s, 1)
    assert not q[:, cols:].any()
    # the same values in float32 in another order at most; a border's other side is a step of e4m3 away, 2^-3 of the value, twice that
    # where the scale is on the other side too
    blocks = -(-cols // 128)
    unit = torch.ldexp(torch.ones(rows, blocks, dtype=torch.float64), want_scale[:, :blocks].int() - 127).repeat_interleave(128, 1)
    assert bool(((got - want).abs() <= 2 * torch.maximum(2.0 ** -3 * want.abs(), 2.0 ** -9 * unit)).all())
    assert float((got != want).double().mean()) <= 0.01
