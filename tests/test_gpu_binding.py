"""What the binding takes of torch tensors, on the GPU."""
import pytest
import torch

from operator_util import randn

pytestmark = pytest.mark.gpu


def test_one_row_of_8_bits_from_a_wider_tensor():
    import paper_2505_16864_amd as J
    x = randn(1, 1, 100).float().cuda()
    want, want_scale = torch.empty((1, 128), dtype=torch.uint8, device="cuda:0"), torch.empty((1, 4), dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm(x, want, y_scale=want_scale, weight_offset=1.0)
    room, scale = torch.full((3, 384), 77, dtype=torch.uint8, device="cuda:0"), torch.full((3, 4), 77, dtype=torch.uint8, device="cuda:0")
    J.jenga_layer_norm(x, room[1:2, 128:256], y_scale=scale[1:2], weight_offset=1.0)
    torch.cuda.synchronize()
    assert torch.equal(room[1:2, 128:256], want) and torch.equal(scale[1:2], want_scale)
    room[1:2, 128:256] = 77
    scale[1:2] = 77
    assert bool((room == 77).all()) and bool((scale == 77).all())


def _pass(J, x):
    """Every call on torch tensors in a row, none told its stream; what they left."""
    def make(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda:0")

    rows, cols = x.shape
    y, mean, rstd, dx, dw, db = make(rows, cols), make(rows), make(rows), make(rows, cols), make(1, cols), make(1, cols)
    ws = make(J.jenga_layer_norm_grad_workspace(rows, cols), dtype=torch.uint8)
    q, s, b, bs = make(rows, cols, dtype=torch.uint8), make(rows, 4, dtype=torch.uint8), make(128, cols, dtype=torch.uint8), make(1, 4, dtype=torch.uint8)
    out, turned = make(rows, 128), make(1, rows, 2, 64)
    cfg, host = J.make_rotary(1, 8, rows // 8, 64, (0, 32, 32)), torch.empty(8 * 32 + rows // 8 * 32)
    J.jenga_rotary_table(cfg, host)
    table = host.cuda()

    def run():
        J.jenga_layer_norm(x, y, mean=mean, rstd=rstd, weight_offset=1.0)
        J.jenga_layer_norm_grad(x, y, dx, None, mean, rstd, dw, db, ws, weight_offset=1.0)
        J.jenga_quantize(y, q, s)
        J.jenga_quantize(y[:128], b, bs, 128)
        J.jenga_matmul(q, s, b, bs, out)
        J.jenga_rotary(cfg, table, out.view(1, rows, 2, 64), turned)
        return [t.clone() for t in (y, dx, dw, db, mean, rstd, q, s, b, bs, out, turned)]

    return run


# On a stream of torch's, behind work that keeps it busy, and captured: the calls are in order with the tensors' own work.
def test_calls_follow_the_current_stream():
    import paper_2505_16864_amd as J
    inputs = [randn(10 + i, 256, 128).float().cuda() for i in range(3)]
    want = [_pass(J, x)() for x in inputs]
    x, busy = inputs[0].clone(), torch.randn((4096, 4096), device="cuda:0")
    run, side = _pass(J, x), torch.cuda.Stream()
    run()
    torch.cuda.synchronize()
    for i in (1, 2, 0):
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy                                  # x is not there before these are done
            x.copy_(inputs[i])
            got = run()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), i
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in (2, 1, 0, 1):
        x.copy_(inputs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), i
        x.copy_(inputs[(i + 1) % 3])
        assert all(torch.equal(a, b) for a, b in zip(run(), want[(i + 1) % 3])), i
