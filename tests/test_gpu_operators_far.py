"""The calls around the attention on tensors whose offsets pass 32 bits, and captured into graphs on a stream of their own.

Large inputs are a small one repeated: every repetition has to give the bits of the first, and the first is checked against float64."""
import pytest
import torch

from operator_util import TYPES, U32, check, half_step, held_values, quantize, randn, rotary

pytestmark = pytest.mark.gpu


def _quantized(x, block_rows):
    import paper_2505_16864_amd as J
    rows, cols = x.shape
    q = torch.empty((rows, J.padded_columns(cols)), dtype=torch.float8_e4m3fn, device="cuda:0")
    scale = torch.empty((-(-rows // block_rows), J.scale_columns(cols)), dtype=torch.uint8, device="cuda:0")
    J.jenga_quantize(x, q, scale, block_rows)
    return q, scale


def _repeated(t, times):
    return t.view(torch.uint8).repeat(times, 1).view(t.dtype)


def _all_like_the_first(t, rows):
    whole = t.view(-1, rows, *t.shape[1:])
    for i in range(1, whole.shape[0]):
        assert torch.equal(whole[i], whole[0]), i


# 4.3e9 values of a, of b and of the result.
@pytest.mark.parametrize("times,rows,n,k,big_b", [(410, 320, 130, 32768, False), (438, 320, 16400, 128, False), (342, 384, 3, 32768, True),
                                                  (342, 384, 20, 32768, True)])
def test_products(times, rows, n, k, big_b):
    import paper_2505_16864_amd as J
    big, big_scale = _quantized(randn(1, rows, k).float().cuda(), 128 if big_b else 1)
    other, other_scale = _quantized(randn(2, n, k).float().cuda(), 1 if big_b else 128)
    many, many_scale = _repeated(big, times), _repeated(big_scale, times)
    A, B = held_values(big, big_scale, 128 if big_b else 1), held_values(other, other_scale, 1 if big_b else 128)
    if big_b:
        out = torch.empty((n, rows * times), dtype=torch.bfloat16, device="cuda:0")
        J.jenga_matmul(other, other_scale, many, many_scale, out)
        out = out.t().contiguous()
    else:
        out = torch.empty((rows * times, n), dtype=torch.bfloat16, device="cuda:0")
        J.jenga_matmul(many, many_scale, other, other_scale, out)
    torch.cuda.synchronize()
    _all_like_the_first(out, rows)
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    check(out[:rows], want, half_step(torch.bfloat16) * want.abs() * 1.01 + (8 * 2.0 ** -13 + U32 * k) * size, "first rows")


def test_rows_of_norm_and_quantisation():
    import paper_2505_16864_amd as J
    times, rows, cols = 2100, 250, 8192
    total = times * rows
    pattern, w = randn(3, rows, cols).to(torch.bfloat16), randn(4, cols).float()
    x = pattern.cuda().repeat(times, 1)
    y, mean, rstd = torch.empty_like(x), torch.empty(total, device="cuda:0"), torch.empty(total, device="cuda:0")
    J.jenga_layer_norm(x, y, w.cuda(), mean=mean, rstd=rstd)
    _all_like_the_first(y, rows)
    X = pattern.double()
    r = 1 / torch.sqrt(X.var(1, unbiased=False, keepdim=True) + 1e-6)
    h = (X - X.mean(1, keepdim=True)) * r
    want = h * w.double()
    slack = U32 * (w.double().abs() * r * 26 * X.abs().mean(1, keepdim=True) + 84 * want.abs())
    check(y[:rows], want, half_step(torch.bfloat16) * want.abs() + slack * 1.01, "y")
    dx, ws = torch.empty_like(x), torch.empty(J.jenga_layer_norm_grad_workspace(total, cols), dtype=torch.uint8, device="cuda:0")
    dw, db = torch.empty(cols, device="cuda:0"), torch.empty(cols, device="cuda:0")
    J.jenga_layer_norm_grad(x, y, dx, w.cuda(), mean, rstd, dw, db, ws)
    torch.cuda.synchronize()
    _all_like_the_first(dx, rows)
    dy = y[:rows].cpu().double()
    h = (X - mean[:rows].cpu().double()[:, None]) * rstd[:rows].cpu().double()[:, None]
    # 256 parts of 2051 rows each, added up in sixteenths: no more than 2100 additions follow each other
    for got, term in ((dw, dy * h), (db, dy)):
        check(got, times * term.sum(0), U32 * 2100 * times * term.abs().sum(0), "sums over the rows")
    g = dy * w.double()
    want = rstd[:rows].cpu().double()[:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    slack = U32 * r * (8 * g.abs() + 150 * g.abs().mean(1, keepdim=True) + h.abs() * 158 * (g * h).abs().mean(1, keepdim=True))
    check(dx[:rows], want, half_step(torch.bfloat16) * want.abs() + slack * 1.01, "dx")
    del y, dx
    q, scale = _quantized(x, 1)
    _all_like_the_first(q.view(torch.uint8), rows)
    _all_like_the_first(scale, rows)
    held, bytes_ = quantize(X, 1)
    assert torch.equal(held_values(q[:rows], scale[:rows], 1), held) and torch.equal(scale[:rows].cpu(), bytes_)


@pytest.mark.parametrize("halves", [False, True])
def test_rotary_in_place(halves):
    import paper_2505_16864_amd as J
    T, H, W, heads, dims = 33, 45, 80, 160, (16, 56, 56)
    cfg = J.make_rotary(T, H, W, 128, dims, flags=J.JENGA_ROTARY_HALVES if halves else 0)
    table = torch.empty(T * dims[0] + H * dims[1] + W * dims[2])
    J.jenga_rotary_table(cfg, table)
    one = randn(5, 1, T * H * W, 1, 128).to(torch.bfloat16)
    x = one.cuda().expand(2, -1, heads, -1).contiguous()
    J.jenga_rotary(cfg, table.cuda(), x, x)
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(heads):
            assert torch.equal(x[b, :, h], x[0, :, 0]), (b, h)
    want = rotary(one.double(), T, H, W, dims, 10000.0, halves=halves)
    # cos and sin are rounded to float32, two products and a sum; a pair's values are at most its length
    check(x[:1, :, :1], want, half_step(torch.bfloat16) * want.abs() + 8 * U32 * one.double().abs().max(), "turned")


# Captured on a stream of its own, replayed with new inputs, eager work of the same calls (with a workspace of its own) between the replays.
@pytest.mark.parametrize("rows,cols,group_rows", [(300, 777, 100), (40, 8200, 40)])
def test_norm_and_gradient_in_a_graph(rows, cols, group_rows):
    import paper_2505_16864_amd as J
    groups = -(-rows // group_rows)
    w, b = randn(6, groups, cols).float().cuda(), randn(7, groups, cols).float().cuda()

    class Pass:
        def __init__(self):
            self.x, self.dy, self.y, self.dx = [torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda:0") for _ in range(4)]
            self.mean, self.rstd = [torch.empty(rows, device="cuda:0") for _ in range(2)]
            self.dw, self.db = [torch.empty((groups, cols), device="cuda:0") for _ in range(2)]
            self.ws = torch.empty(J.jenga_layer_norm_grad_workspace(rows, cols, group_rows), dtype=torch.uint8, device="cuda:0")

        def run(self):
            stream = torch.cuda.current_stream().cuda_stream
            J.jenga_layer_norm(self.x, self.y, w, b, mean=self.mean, rstd=self.rstd, group_rows=group_rows, weight_offset=1.0, stream=stream)
            J.jenga_layer_norm_grad(self.x, self.dy, self.dx, w, self.mean, self.rstd, self.dw, self.db, self.ws, group_rows=group_rows,
                                    weight_offset=1.0, stream=stream)

        def results(self):
            return [t.clone() for t in (self.y, self.dx, self.dw, self.db, self.mean, self.rstd)]

    eager, caught = Pass(), Pass()
    inputs = [[randn(10 + 2 * i + j, rows, cols).to(torch.bfloat16).cuda() for j in range(2)] for i in range(3)]
    want = []
    for x, dy in inputs:
        eager.x.copy_(x), eager.dy.copy_(dy)
        eager.run()
        want.append(eager.results())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught.run()
    side = torch.cuda.Stream()
    for i in (2, 0, 1, 2, 1):
        caught.x.copy_(inputs[i][0]), caught.dy.copy_(inputs[i][1])
        eager.x.copy_(inputs[(i + 1) % 3][0]), eager.dy.copy_(inputs[(i + 1) % 3][1])
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager.run()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(caught.results(), want[i])), i
        assert all(torch.equal(a, c) for a, c in zip(eager.results(), want[(i + 1) % 3])), i


# Products of every kind of kernel in one graph: no tiles, tiles in two groups, tiles of each size, float32 results; quantisation in front.
def test_products_in_a_graph():
    import paper_2505_16864_amd as J
    sizes = [(3, 200, 640, "bf16"), (60, 300, 640, "f32"), (200, 5000, 384, "f16"), (1300, 2600, 512, "f32"), (9000, 9000, 256, "bf16")]
    work = []
    for i, (m, n, k, out) in enumerate(sizes):
        b, b_scale = _quantized(randn(30 + i, n, k).float().cuda(), 128)
        x = [randn(40 + 3 * i + j, m, k).float().cuda() for j in range(3)]
        a, a_scale = _quantized(x[0], 1)
        work.append((x, x[0].clone(), a, a_scale, b, b_scale, torch.empty((m, n), dtype=TYPES[out], device="cuda:0")))

    def run(which=None):
        stream = torch.cuda.current_stream().cuda_stream
        for x, now, a, a_scale, b, b_scale, out in work:
            J.jenga_quantize(now if which is None else x[which], a, a_scale, stream=stream)
            J.jenga_matmul(a, a_scale, b, b_scale, out, stream=stream)

    want = []
    for i in range(3):
        run(i)
        want.append([w[-1].clone() for w in work])
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
