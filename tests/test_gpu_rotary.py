"""jenga_rotary against float64, through the C ABI.

Tolerance: cos and sin are float64 values rounded to float32 (u = 2^-24 of a number of at most 1 each), two products and a sum are
float32: at most 4 u (|x| + |y|) of the pair, and one rounding to the tensor's type."""
import pytest
import torch

import jenga_inputs as ji
from operator_util import TYPES, U32, check, half_step, randn, rotary

pytestmark = pytest.mark.gpu

# head_dim, channels of the axes
HEADS = [(128, (16, 56, 56)), (128, (44, 42, 42)), (64, (16, 24, 24)), (64, (20, 22, 22)), (64, (0, 32, 32)), (72, (16, 16, 20)),
         (96, (32, 32, 32)), (128, (16, 32, 48)), (2, (2, 0, 0)), (10, (2, 4, 2)), (256, (64, 96, 96)), (8, (0, 2, 0))]


def _cfg(J, grid, head_dim, dims, halves, inverse=False, theta=10000.0, origin=(0, 0, 0), step=(1, 1, 1)):
    flags = (J.JENGA_ROTARY_HALVES if halves else 0) | (J.JENGA_ROTARY_INVERSE if inverse else 0)
    cfg = J.make_rotary(*grid, head_dim, dims, theta, origin, step, flags)
    table = torch.empty(grid[0] * dims[0] + grid[1] * dims[1] + grid[2] * dims[2], dtype=torch.float32)
    J.jenga_rotary_table(cfg, table)
    return cfg, table.cuda()


def _tolerance(x, want, dtype):
    """4 u of the sum of magnitudes of the channels that a value may be paired with, at most the head's two largest."""
    top = x.abs().topk(min(2, x.shape[-1]), dim=-1).values.sum(-1, keepdim=True)
    return half_step(dtype) * want.abs() + 4 * U32 * top * 1.01 + (2.0 ** -25 if dtype == torch.float16 else 0)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("head_dim,dims", HEADS)
def test_grid_order(head_dim, dims, dtype, halves):
    import paper_2505_16864_amd as J
    grid, n_text, batch = (3, 5, 7), 9, 2
    for inverse in (False, True):
        cfg, table = _cfg(J, grid, head_dim, dims, halves, inverse, 256.0, (0.5, 0, -3), (1, 0.75, 1.25))
        tokens = 105 + n_text
        q, k = randn(1, batch, tokens, 5, head_dim).to(TYPES[dtype]), randn(2, batch, tokens, 3, head_dim).to(TYPES[dtype])
        out = [torch.full_like(t, 7.0, device="cuda:0") for t in (q, k)]
        J.jenga_rotary(cfg, table, q.cuda(), out[0], k.cuda(), out[1])
        torch.cuda.synchronize()
        for x, got in ((q, out[0]), (k, out[1])):
            want = rotary(x.double(), *grid, dims, 256.0, (0.5, 0, -3), (1, 0.75, 1.25), halves, inverse)
            check(got, want, _tolerance(x.double(), want, x.dtype), "inverse" if inverse else "forward")
            assert torch.equal(got[:, 105:].cpu(), x[:, 105:])       # text keeps its bits
            kept = sum(dims)
            assert torch.equal(got[..., kept:].cpu(), x[..., kept:])


@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 300])
@pytest.mark.parametrize("halves", [False, True])
def test_token_counts(tokens, halves):
    import paper_2505_16864_amd as J
    cfg, table = _cfg(J, (4, 8, 8), 64, (16, 24, 24), halves)
    q = randn(tokens, 1, tokens, 1, 64).to(torch.bfloat16)
    out = torch.full_like(q, 7.0, device="cuda:0")
    J.jenga_rotary(cfg, table, q.cuda(), out)
    torch.cuda.synchronize()
    want = rotary(q.double(), 4, 8, 8, (16, 24, 24), 10000.0, halves=halves)
    check(out, want, _tolerance(q.double(), want, q.dtype))


# Q and K as columns of one product, in place and not, addresses off the 16-byte grid, V between them untouched.
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("head_dim,dims", [(64, (16, 24, 24)), (128, (44, 42, 42)), (10, (2, 4, 2)), (72, (16, 16, 20))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_columns_of_one_product_in_place(head_dim, dims, dtype, halves):
    import paper_2505_16864_amd as J
    cfg, table = _cfg(J, (2, 3, 5), head_dim, dims, halves)
    heads, batch, tokens = 12, 2, 33
    for shift in (0, 1):
        data = randn(5, batch, tokens, 3, heads, head_dim).to(TYPES[dtype])
        room = torch.zeros(data.numel() + 8, dtype=data.dtype, device="cuda:0")
        qkv = room[shift:shift + data.numel()].view(data.shape)
        qkv.copy_(data)
        q, v, k = qkv.unbind(2)
        apart = [torch.empty((batch, tokens, heads, head_dim), dtype=data.dtype, device="cuda:0") for _ in range(2)]
        J.jenga_rotary(cfg, table, q, apart[0], k, apart[1])
        J.jenga_rotary(cfg, table, q, q, k, k)
        torch.cuda.synchronize()
        for i, got in ((0, q), (2, k)):
            x = data[:, :, i].double()
            want = rotary(x, 2, 3, 5, dims, 10000.0, halves=halves)
            check(got, want, _tolerance(x, want, data.dtype))
        assert torch.equal(q, apart[0]) and torch.equal(k, apart[1]) and torch.equal(v.cpu(), data[:, :, 1])
        assert bool((room[:shift] == 0).all()) and bool((room[shift + data.numel():] == 0).all())


# Curve side: the cells of a plan's tokens, text and pads as they are.
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("name", ["tiny", "small"])
def test_curve_order(name, halves):
    import paper_2505_16864_amd as J
    w = dict(ji.WORKLOADS[name], batch=2, n_text=ji.WORKLOADS[name]["n_text"] + 5)
    D = w["head_dim"]
    dims = (D // 4, D // 4 + 8, D // 2 - 8)
    cfg, table = _cfg(J, (w["T"], w["H"], w["W"]), D, dims, halves, theta=256.0)
    plan = J.jenga_plan_create(J.make_config(w["T"], w["H"], w["W"], w["n_text"], 2, w["heads"], D, w["block"], w["topk"], w["p"]))
    try:
        info = J.jenga_plan_info(plan)
        q = ji.make_qkv(w, 12)[0].cuda()
        curve = torch.empty((2, w["heads"], info.N_pad, D), dtype=torch.bfloat16, device="cuda:0")
        turned = torch.empty_like(q)
        J.jenga_rotary(cfg, table, q, turned)                       # turn, then re-order
        J.jenga_curve_permute(plan, turned, curve)
        again = torch.empty_like(curve)
        J.jenga_curve_permute(plan, q, again)                       # re-order, then turn
        view = again.transpose(1, 2)
        J.jenga_rotary(cfg, table, view, view, plan=plan)
        torch.cuda.synchronize()
    finally:
        J.jenga_plan_destroy(plan)
    assert torch.equal(curve, again)


# Sequences of several grids, a padded batch: cells by token, axes that stay, cells past the end.
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("head_dim,dims", [(64, (16, 24, 24)), (128, (44, 42, 42)), (10, (2, 4, 2))])
def test_cells_by_token(head_dim, dims, halves):
    import paper_2505_16864_amd as J
    cfg, table = _cfg(J, (3, 6, 8), head_dim, dims, halves)
    gen = torch.Generator().manual_seed(3)
    cells = torch.stack([torch.randint(-2, n + 3, (2, 50), generator=gen) for n in (3, 6, 8)], -1).int()
    q = randn(8, 2, 50, 4, head_dim).to(torch.bfloat16)
    out = torch.empty_like(q, device="cuda:0")
    J.jenga_rotary(cfg, table, q.cuda(), out, cells=cells.cuda())
    torch.cuda.synchronize()
    want = rotary(q.double(), 3, 6, 8, dims, 10000.0, halves=halves, cells=cells.long())
    check(out, want, _tolerance(q.double(), want, q.dtype))


# Far positions: the angles come from float64.  The gradient is the inverse turn: <dy, R x> = <R^T dy, x>, and there and back is x.
@pytest.mark.parametrize("halves", [False, True])
def test_far_positions_and_the_gradient(halves):
    import paper_2505_16864_amd as J
    origin, step = (1.0e6, 12345.0, 0.0), (1.0, 3.0, 1000.0)
    cfg, table = _cfg(J, (2, 4, 5), 64, (16, 24, 24), halves, origin=origin, step=step)
    back, _ = _cfg(J, (2, 4, 5), 64, (16, 24, 24), halves, inverse=True, origin=origin, step=step)
    x, dy = randn(1, 1, 40, 3, 64).float(), randn(2, 1, 40, 3, 64).float()
    y, dx, again = [torch.empty_like(x, device="cuda:0") for _ in range(3)]
    J.jenga_rotary(cfg, table, x.cuda(), y)
    J.jenga_rotary(back, table, dy.cuda(), dx)
    J.jenga_rotary(back, table, y, again)
    torch.cuda.synchronize()
    want = rotary(x.double(), 2, 4, 5, (16, 24, 24), 10000.0, origin, step, halves)
    check(y, want, _tolerance(x.double(), want, x.dtype))
    check(again, x.double(), 3 * _tolerance(x.double(), x.double(), x.dtype))
    grad = torch.zeros_like(x, dtype=torch.float64)
    # differences along every channel of one head; the map is linear, so a difference of any width is exact
    base = rotary(torch.zeros(1, 40, 3, 64, dtype=torch.float64), 2, 4, 5, (16, 24, 24), 10000.0, origin, step, halves)
    for c in range(64):
        e = torch.zeros(1, 40, 3, 64, dtype=torch.float64)
        e[..., c] = 1.0
        moved = rotary(e, 2, 4, 5, (16, 24, 24), 10000.0, origin, step, halves) - base
        grad[..., c] = (moved * dy.double()).sum(-1)
    check(dx, grad, _tolerance(dy.double(), grad, x.dtype))


def test_many_tokens_one_head():
    import paper_2505_16864_amd as J
    cfg, table = _cfg(J, (33, 45, 80), 64, (16, 24, 24), False)
    q = torch.randn((1, 118800, 1, 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    out = torch.empty_like(q, device="cuda:0")
    J.jenga_rotary(cfg, table, q.cuda(), out)
    torch.cuda.synchronize()
    want = rotary(q.double(), 33, 45, 80, (16, 24, 24), 10000.0)
    check(out, want, _tolerance(q.double(), want, q.dtype))


def test_no_tokens():
    import paper_2505_16864_amd as J
    cfg, table = _cfg(J, (2, 2, 2), 64, (16, 24, 24), False)
    q = torch.empty((1, 0, 3, 64), dtype=torch.bfloat16, device="cuda:0")
    J.jenga_rotary(cfg, table, q, q)
    torch.cuda.synchronize()
    assert q.numel() == 0
