"""Layer norm's gradient where mean and 1 / spread are so far apart that (0 - mean) * rstd is no float32: values that are not there (columns
behind a row's last one, rows behind the last one) have to stay out of every sum.

A row whose values are all 2^120 has mean 2^120 exactly (up to 255 of them add up below 2^128, a power of two times a whole number), no
spread, h = 0 and rstd = 1 / sqrt(eps) = 2^10 for eps = 2^-20.  So dx = rstd (g - mean(g)), dweight = 0 and dbias = the sum of dy."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, randn

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
