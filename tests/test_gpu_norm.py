"""jenga_layer_norm and its gradient against float64, through the C ABI.

Tolerances.  u = 2^-24.  A sum of n float32 values in any order is off by at most n u times the sum of their magnitudes; in the forward
kernel at most 26 additions follow each other for the mean and 136 for the squares (16 pieces of eight values a lane, six steps across
the wavefront; rows too long for that: 16 turns, 10 steps).  So mean is off by 26 u mean|x|, r by half of 140 u, and y by
|w| r 26 u mean|x| + 80 u |h w| + 4 u (|h w| + |b|) before it is rounded once."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, held_values, quantize, randn

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _inputs(rows, cols, groups, dtype, params, seed, offset=0.7):
    x = (randn(seed, rows, cols) * (0.5 + randn(seed + 1, cols).abs()) + offset * randn(seed + 2, cols)).to(TYPES[dtype])
    w = (0.5 * randn(seed + 3, groups, cols)).to(TYPES[params])
    b = (0.5 * randn(seed + 4, groups, cols)).to(TYPES[params])
    return x, w, b


def _plain(x, w, b, group_rows, w0, eps=EPS):
    x = x.double()
    group = torch.arange(x.shape[0]) // group_rows
    mean = x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * r
    w = (w0 + w.double())[group] if w is not None else torch.full_like(x, w0)
    b = b.double()[group] if b is not None else torch.zeros_like(x)
    y = h * w + b
    slack = U32 * (w.abs() * r * 26 * x.abs().mean(1, keepdim=True) + 84 * (h * w).abs() + 4 * b.abs())
    return y, slack, mean[:, 0], r[:, 0], h, w


SIZES = [(1, 1), (1, 2), (3, 7), (5, 8), (4, 64), (2, 127), (7, 128), (6, 129), (9, 512), (5, 513), (33, 777), (3, 1536), (2, 2047),
         (4, 2048), (3, 2049), (2, 4000), (5, 5120), (2, 5121), (3, 8192), (2, 8193), (2, 20000), (1, 131072), (260, 96)]


@pytest.mark.parametrize("dtype,params", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype, params):
    import paper_2505_16864_amd as J
    x, w, b = _inputs(rows, cols, 1, dtype, params, 10 * rows + cols)
    want, slack, mean, r, _, _ = _plain(x, w, b, rows, 1.0)
    y = torch.full((rows, cols), 7.0, dtype=x.dtype, device="cuda:0")
    stats = [torch.full((rows,), 7.0, device="cuda:0") for _ in range(2)]
    J.jenga_layer_norm(x.cuda(), y, w.cuda(), b.cuda(), mean=stats[0], rstd=stats[1], weight_offset=1.0, eps=EPS)
    torch.cuda.synchronize()
    check(y, want, half_step(x.dtype) * want.abs() + slack * (1 + half_step(x.dtype)) + (2.0 ** -25 if dtype == "f16" else 0), "y")
    check(stats[0], mean, 26 * U32 * x.double().abs().mean(1) + U32 * mean.abs(), "mean")
    check(stats[1], r, (75 * U32 + 26 * U32 * r * x.double().abs().mean(1)) * r, "rstd")


# Groups of rows (the last one short), rows and groups that lie apart, weight or bias alone, in place, outputs that lie between.
@pytest.mark.parametrize("rows,cols,group_rows", [(10, 96, 4), (7, 1000, 1), (12, 640, 5), (3, 8200, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_and_strides(rows, cols, group_rows, dtype):
    import paper_2505_16864_amd as J
    groups = -(-rows // group_rows)
    x, w, b = _inputs(rows, cols, groups, dtype, dtype, 77 + rows)
    want, slack, _, _, _, _ = _plain(x, w, b, group_rows, 1.0)
    room = torch.full((rows, 2 * cols + 5), 3.0, dtype=x.dtype, device="cuda:0")
    room[:, :cols] = x.cuda()
    params = torch.zeros((groups, 3 * cols + 1), dtype=x.dtype, device="cuda:0")     # scale and shift among other vectors
    params[:, 1:1 + cols], params[:, 2 * cols:3 * cols] = w.cuda(), b.cuda()
    pw, pb = params[:, 1:1 + cols], params[:, 2 * cols:3 * cols]
    y = room[:, cols + 3:2 * cols + 3]
    J.jenga_layer_norm(room[:, :cols], y, pw, pb, group_rows=group_rows, weight_offset=1.0, eps=EPS)
    torch.cuda.synchronize()
    tol = lambda t, s: half_step(x.dtype) * t.abs() + s * 1.01  # noqa: E731
    check(y, want, tol(want, slack), "strided")
    assert torch.equal(room[:, :cols].cpu(), x) and bool((room[:, cols:cols + 3] == 3).all()) and bool((room[:, 2 * cols + 3:] == 3).all())
    for ww, bb in ((w, None), (None, b), (None, None)):
        want, slack, _, _, _, _ = _plain(x, ww, bb, group_rows, 0.5)
        again = x.cuda()
        J.jenga_layer_norm(again, again, ww.cuda() if ww is not None else None, bb.cuda() if bb is not None else None,
                           group_rows=group_rows, weight_offset=0.5, eps=EPS)
        torch.cuda.synchronize()
        check(again, want, tol(want, slack), "in place")


# A row that is constant, one far off zero, one with an infinity, one with a NaN; the others keep their values.
@pytest.mark.parametrize("cols", [96, 3000, 9000])
def test_rows_without_spread_and_rows_that_are_not_finite(cols):
    import paper_2505_16864_amd as J
    x = randn(5, 6, cols).float()
    x[1] = 2.5
    x[2] += 4096.0
    x[3, cols // 2] = float("inf")
    x[4, cols - 1] = float("nan")
    y = torch.empty(6, cols, device="cuda:0")
    J.jenga_layer_norm(x.cuda(), y, eps=EPS, weight_offset=1.0)
    torch.cuda.synchronize()
    want, slack, _, _, _, _ = _plain(x, None, None, 6, 1.0)
    got = y.cpu()
    assert bool((got[1] == 0).all())
    assert bool(torch.isnan(got[3]).any()) and bool(torch.isnan(got[4]).all())
    for i in (0, 2, 5):
        check(got[i], want[i], U32 * want[i].abs() + slack[i], "row %d" % i)


# Results straight to 8 bits.  A float32 result off by the slack may fall on the other side of a border between two e4m3 values,
# and the largest of a block on the other side of a border between two scales: then the value is the neighbour's, one step of
# 2^-3 of the value (2^-9 of the unit among the smallest) further.
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 128), (5, 130), (4, 1000), (33, 1536), (2, 5120), (2, 8192), (3, 9000)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_eight_bit_result(rows, cols, dtype):
    import paper_2505_16864_amd as J
    x, w, b = _inputs(rows, cols, 1, dtype, dtype, 31 + cols)
    y, slack, _, _, _, _ = _plain(x, w, b, rows, 1.0)
    q = torch.full((rows, J.padded_columns(cols)), 99, dtype=torch.uint8, device="cuda:0")
    scale = torch.full((rows, J.scale_columns(cols)), 99, dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm(x.cuda(), q, w.cuda(), b.cuda(), y_scale=scale, weight_offset=1.0, eps=EPS)
    torch.cuda.synchronize()
    want, want_scale = quantize(y, 1)
    got = held_values(q, scale, 1)
    assert bool((q[:, cols:] == 0).all())
    blocks = -(-cols // 128)
    assert bool((scale[:, blocks:] == 0).all())
    unit = torch.ldexp(torch.ones(rows, blocks, dtype=torch.float64), want_scale[:, :blocks].int() - 127).repeat_interleave(128, 1)
    full, room = torch.zeros_like(want), torch.zeros_like(want)
    full[:, :cols], room[:, :cols] = y, slack * 1.01
    step = torch.maximum(2.0 ** -3 * full.abs(), 2.0 ** -9 * unit) * 2     # the coarser of the two scales
    off = (got - full).abs()
    assert bool((off <= step / 2 + room).all()), float((off - step / 2 - room).max())
    same = got == want
    assert float((~same).double().mean()) <= 0.01 and (scale.cpu() != want_scale).double().mean() <= 0.05


def _grads(x, dy, w, mean, rstd, group_rows, w0):
    """The formulas in float64 from the float32 statistics, and how far float32 sums may be off."""
    x, dy, mean, rstd = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    rows = x.shape[0]
    group = torch.arange(rows) // group_rows
    h = (x - mean) * rstd
    wide = (w0 + w.double())[group] if w is not None else torch.full_like(x, w0)
    g = dy * wide
    mg, mgh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = rstd * (g - mg - h * mgh)
    # at most 140 additions follow each other for either mean
    slack = U32 * rstd * (8 * g.abs() + 150 * g.abs().mean(1, keepdim=True) + h.abs() * (150 * (g * h).abs().mean(1, keepdim=True) + 8 * mgh.abs()))
    groups = -(-rows // group_rows)
    sums = []
    for term in (dy * h, dy):
        total = torch.zeros((groups, x.shape[1]), dtype=torch.float64).index_add_(0, group, term)
        size = torch.zeros_like(total).index_add_(0, group, term.abs())
        sums.append((total, U32 * (min(rows, group_rows) + 8) * size))
    return dx, slack, sums


@pytest.mark.parametrize("dtype,params", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols,group_rows", [(1, 1, 1), (3, 7, 3), (9, 130, 4), (40, 512, 40), (65, 777, 65), (21, 1536, 10),
                                                  (70, 2048, 70), (5, 2500, 2), (19, 4096, 19), (6, 5120, 6), (11, 8192, 11),
                                                  (5, 8200, 2), (600, 40, 150), (1030, 24, 1)])
def test_gradient(rows, cols, group_rows, dtype, params):
    import paper_2505_16864_amd as J
    groups = -(-rows // group_rows)
    x, w, _ = _inputs(rows, cols, groups, dtype, params, 500 + rows + cols)
    dy = randn(900 + rows, rows, cols).to(x.dtype)
    gx, gw = x.cuda(), w.cuda()
    y = torch.empty_like(gx)
    mean, rstd = torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
    J.jenga_layer_norm(gx, y, gw, None, mean=mean, rstd=rstd, group_rows=group_rows, weight_offset=1.0, eps=EPS)
    dx = torch.full_like(gx, 7.0)
    dw, db = [torch.full((groups, cols), 7.0, device="cuda:0") for _ in range(2)]
    ws = torch.full((J.jenga_layer_norm_grad_workspace(rows, cols, group_rows),), 0xFF, dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm_grad(gx, dy.cuda(), dx, gw, mean, rstd, dw, db, ws, group_rows=group_rows, weight_offset=1.0)
    torch.cuda.synchronize()
    want, slack, sums = _grads(x, dy, w, mean.cpu(), rstd.cpu(), group_rows, 1.0)
    check(dx, want, half_step(x.dtype) * want.abs() + slack * 1.01 + (2.0 ** -25 if dtype == "f16" else 0), "dx")
    check(dw, sums[0][0], sums[0][1], "dweight")
    check(db, sums[1][0], sums[1][1], "dbias")
    # one gradient of the two, none of them, no weight
    for a, b in ((dw, None), (None, db), (None, None)):
        for t in (a, b):
            if t is not None:
                t.fill_(7.0)
        dx.fill_(7.0)
        J.jenga_layer_norm_grad(gx, dy.cuda(), dx, None, mean, rstd, a, b, ws if a is not None or b is not None else None,
                                group_rows=group_rows, weight_offset=0.25)
        torch.cuda.synchronize()
        want, slack, sums = _grads(x, dy, None, mean.cpu(), rstd.cpu(), group_rows, 0.25)
        check(dx, want, half_step(x.dtype) * want.abs() + slack * 1.01 + (2.0 ** -25 if dtype == "f16" else 0), "dx without a weight")
        for t, (total, tol) in ((a, sums[0]), (b, sums[1])):
            if t is not None:
                check(t, total, tol, "one gradient")


# Against differences of the float64 forward pass: (y(x + e d) - y(x - e d)) / 2e along a direction, times dy, is dx . d up to e^2.
@pytest.mark.parametrize("rows,cols,group_rows", [(6, 96, 2), (3, 2500, 3)])
def test_gradient_against_differences(rows, cols, group_rows):
    import paper_2505_16864_amd as J
    groups = -(-rows // group_rows)
    x, w, b = _inputs(rows, cols, groups, "f32", "f32", 41)
    dy = randn(42, rows, cols).float()
    gx, gw = x.cuda(), w.cuda()
    y, mean, rstd = torch.empty_like(gx), torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
    J.jenga_layer_norm(gx, y, gw, b.cuda(), mean=mean, rstd=rstd, group_rows=group_rows, weight_offset=1.0, eps=EPS)
    dx, dw, db = torch.empty_like(gx), torch.empty(groups, cols, device="cuda:0"), torch.empty(groups, cols, device="cuda:0")
    ws = torch.empty(J.jenga_layer_norm_grad_workspace(rows, cols, group_rows), dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm_grad(gx, dy.cuda(), dx, gw, mean, rstd, dw, db, ws, group_rows=group_rows, weight_offset=1.0)
    torch.cuda.synchronize()
    f = lambda X, W, B: (_plain(X, W, B, group_rows, 1.0)[0] * dy.double()).sum()  # noqa: E731
    e = 1e-4
    for name, got, at in (("x", dx, 0), ("weight", dw, 1), ("bias", db, 2)):
        args = [x.double(), w.double(), b.double()]
        d = randn(43 + at, *args[at].shape)
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + e * d, args[at] - e * d
        want = float((f(*up) - f(*down)) / (2 * e))
        have = float((got.cpu().double() * d).sum())
        # e^2 times a third derivative of order |dy| r^3, and float32 sums
        size = float((got.cpu().double() * d).abs().sum())
        assert abs(have - want) <= 1e-5 * size + 1e-6 * rows * cols, (name, have, want, size)


def test_strided_gradient_and_the_same_bits_again():
    import paper_2505_16864_amd as J
    rows, cols = 300, 640
    x, w, _ = _inputs(rows, cols, 1, "bf16", "f32", 61)
    dy = randn(62, rows, cols).to(torch.bfloat16)
    both = torch.zeros((rows, 2, cols + 8), dtype=torch.bfloat16, device="cuda:0")
    both[:, 0, :cols] = x.cuda()
    gx, dx = both[:, 0, :cols], both[:, 1, :cols]
    gdy = torch.zeros((rows, cols + 1), dtype=torch.bfloat16, device="cuda:0")
    gdy[:, 1:] = dy.cuda()
    mean, rstd = torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda:0")
    J.jenga_layer_norm(gx, y, w.cuda(), mean=mean, rstd=rstd, eps=EPS)
    results = []
    ws = torch.empty(J.jenga_layer_norm_grad_workspace(rows, cols), dtype=torch.uint8, device="cuda:0")
    for _ in range(2):
        ws.fill_(0xFF)
        dw, db = torch.empty(1, cols, device="cuda:0"), torch.empty(1, cols, device="cuda:0")
        J.jenga_layer_norm_grad(gx, gdy[:, 1:], dx, w.cuda(), mean, rstd, dw, db, ws)
        torch.cuda.synchronize()
        results.append((dx.clone(), dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    want, slack, sums = _grads(x, dy, w, mean.cpu(), rstd.cpu(), rows, 0.0)
    check(dx, want, half_step(torch.bfloat16) * want.abs() + slack * 1.01, "dx")
    check(dw, sums[0][0], sums[0][1], "dweight")
    assert bool((both[:, :, cols:] == 0).all()) and torch.equal(gx.cpu(), x)


def test_no_rows():
    import paper_2505_16864_amd as J
    x = torch.empty((0, 64), device="cuda:0")
    J.jenga_layer_norm(x, torch.empty_like(x), torch.ones(64, device="cuda:0"))
    stats = torch.empty(0, device="cuda:0")
    J.jenga_layer_norm_grad(x, x, torch.empty_like(x), None, stats, stats)
    torch.cuda.synchronize()
