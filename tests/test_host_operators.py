"""CPU tests of the calls around the attention: what they refuse, before any device is touched, and the rotary table."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2505_16864_amd as J

BF16, F16, F32, E4M3 = range(4)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -3
A = 1 << 20          # addresses that no call gets to read: every call here is refused, or has nothing to do
NAN, INF = float("nan"), float("inf")


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(J.jenga_norm_config) == 64 and J.jenga_norm_config.cols.offset == 40
    assert ctypes.sizeof(J.jenga_matmul_config) == 32 and J.jenga_matmul_config.n.offset == 16
    assert ctypes.sizeof(J.jenga_rotary_config) == 96 and J.jenga_rotary_config.theta.offset == 32
    assert ctypes.sizeof(J.jenga_rotary_tensor) == 72 and J.jenga_rotary_tensor.heads.offset == 64


def norm(call="forward", **over):
    a = dict(rows=4, group_rows=4, x_stride=64, y_stride=64, param_stride=64, cols=64, x_type=BF16, y_type=BF16, param_type=BF16,
             eps=1e-6, weight_offset=0.0, x=A, dy=2 * A, weight=3 * A, bias=4 * A, y=5 * A, y_scale=None, mean=6 * A, rstd=7 * A,
             dx=5 * A, dweight=8 * A, dbias=9 * A, ws=16 * A, ws_bytes=1 << 40)
    a.update(over)
    cfg = J.jenga_norm_config(*[a[n] for n, _ in J.jenga_norm_config._fields_])
    if call == "forward":
        return J.raw().jenga_layer_norm(ctypes.byref(cfg), a["x"], a["weight"], a["bias"], a["y"], a["y_scale"], a["mean"],
                                        a["rstd"], None)
    return J.raw().jenga_layer_norm_grad(ctypes.byref(cfg), a["x"], a["dy"], a["weight"], a["mean"], a["rstd"], a["dx"], a["dweight"],
                                         a["dbias"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(group_rows=0), EINVAL),
    (dict(x_stride=63), EINVAL), (dict(y_stride=63), EINVAL), (dict(param_stride=63), EINVAL), (dict(x_type=9), EINVAL),
    (dict(x_type=E4M3), EINVAL), (dict(y_type=-1), EINVAL), (dict(param_type=E4M3), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=NAN), EINVAL), (dict(eps=INF), EINVAL), (dict(weight_offset=NAN), EINVAL), (dict(y_type=F32), EUNSUPPORTED),
    (dict(param_type=F16), EUNSUPPORTED), (dict(cols=1 << 18, x_stride=1 << 18, y_stride=1 << 18, param_stride=1 << 18), EUNSUPPORTED),
    (dict(rows=1 << 41), EUNSUPPORTED), (dict(rows=1 << 40, x_stride=1 << 40), EUNSUPPORTED),
    (dict(y_scale=10 * A), EINVAL), (dict(y_type=E4M3), EINVAL), (dict(y_type=E4M3, y_scale=10 * A), EINVAL),
    (dict(y_type=E4M3, y_scale=10 * A, y_stride=128, y=5 * A + 8), EINVAL), (dict(y_type=E4M3, y_scale=10 * A + 1, y_stride=128), EINVAL),
    (dict(x=A + 1), EINVAL), (dict(y=5 * A + 1), EINVAL), (dict(weight=3 * A + 1), EINVAL), (dict(mean=6 * A + 2), EINVAL),
    (dict(y=A + 2), EINVAL), (dict(y=A + 64 * 2 * 3 + 126), EINVAL), (dict(y=A, y_stride=65), EINVAL), (dict(y=3 * A), EINVAL),
    (dict(mean=5 * A), EINVAL), (dict(mean=7 * A), EINVAL), (dict(rstd=A), EINVAL),
])
def test_norm_refuses(bad, status):
    assert norm(**bad) == status
    if "y" not in bad and "y_scale" not in bad and bad.get("y_type") != E4M3 and "mean" not in bad and "rstd" not in bad:
        assert norm("grad", **bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(mean=None), EINVAL), (dict(rstd=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws=16 * A + 8), EINVAL), (dict(ws_bytes=(1024 + 1) * 64 * 8 - 1), EWORKSPACE), (dict(y_type=E4M3), EUNSUPPORTED),
    (dict(dx=A), EINVAL), (dict(dx=2 * A), EINVAL), (dict(dweight=9 * A), EINVAL), (dict(dweight=5 * A), EINVAL),
    (dict(dbias=16 * A + 256), EINVAL), (dict(dweight=8 * A + 1), EINVAL), (dict(rows=(1 << 20) + 1, group_rows=1), EUNSUPPORTED),
])
def test_norm_gradient_refuses(bad, status):
    assert norm("grad", **bad) == status


def test_norm_without_rows_needs_no_device():
    assert norm(rows=0) == OK and norm("grad", rows=0) == OK


def test_norm_gradient_workspace():
    assert J.jenga_layer_norm_grad_workspace(100, 64) == 1025 * 64 * 8
    assert J.jenga_layer_norm_grad_workspace(100, 64, 30) == (1024 + 4) * 64 * 8
    with pytest.raises(J.JengaError) as e:
        J.jenga_layer_norm_grad_workspace(1 << 21, 64, 1)
    assert e.value.status == EUNSUPPORTED


# Columns of one matrix lie between each other's rows: disjoint, though their spans are not.  (A workspace that is too small is looked at
# last, so that no call gets past its checks.)
def test_columns_of_one_matrix_do_not_overlap():
    inside = dict(rows=4, x_stride=200, weight=None, ws_bytes=0)
    assert norm("grad", x=A, dx=A + 2 * 70, **inside) == EWORKSPACE
    assert norm("grad", x=A + 2 * 130, dx=A, **inside) == EWORKSPACE
    assert norm("grad", x=A, dx=A + 2 * 63, **inside) == EINVAL          # they share a column
    assert norm("grad", x=A, dx=A + 2 * 137, **inside) == EINVAL         # the rows of dx run into the next rows of x


def quantize(**over):
    a = dict(x=A, x_stride=64, x_type=BF16, rows=4, cols=64, block_rows=1, q=2 * A, scale=3 * A)
    a.update(over)
    return J.raw().jenga_quantize(a["x"], a["x_stride"], a["x_type"], a["rows"], a["cols"], a["block_rows"], a["q"], a["scale"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(scale=None), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL),
    (dict(x_stride=63), EINVAL), (dict(block_rows=64), EINVAL), (dict(x_type=E4M3), EINVAL), (dict(x=A + 1), EINVAL),
    (dict(q=2 * A + 8), EINVAL), (dict(scale=3 * A + 2), EINVAL), (dict(q=A), EINVAL), (dict(scale=2 * A + 16), EINVAL),
    (dict(scale=A + 8), EINVAL), (dict(cols=1 << 18, x_stride=1 << 18), EUNSUPPORTED), (dict(rows=(1 << 30) + 1), EUNSUPPORTED),
])
def test_quantize_refuses(bad, status):
    assert quantize(**bad) == status


def matmul(**over):
    a = dict(m=4, out_stride=64, n=64, k=256, out_type=BF16, reserved=0, a=A, a_scale=2 * A, b=3 * A, b_scale=4 * A, bias=5 * A, out=6 * A)
    a.update(over)
    cfg = J.jenga_matmul_config(*[a[n] for n, _ in J.jenga_matmul_config._fields_])
    return J.raw().jenga_matmul(ctypes.byref(cfg), a["a"], a["a_scale"], a["b"], a["b_scale"], a["bias"], a["out"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(a=None), EINVAL), (dict(a_scale=None), EINVAL), (dict(b=None), EINVAL), (dict(b_scale=None), EINVAL), (dict(out=None), EINVAL),
    (dict(m=-1), EINVAL), (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(k=200), EINVAL), (dict(out_stride=63), EINVAL),
    (dict(reserved=1), EINVAL), (dict(out_type=E4M3), EINVAL), (dict(a=A + 8), EINVAL), (dict(b=3 * A + 1), EINVAL),
    (dict(a_scale=2 * A + 2), EINVAL), (dict(bias=5 * A + 2), EINVAL), (dict(out=6 * A + 1), EINVAL), (dict(out=A), EINVAL),
    (dict(out=3 * A + 16), EINVAL), (dict(out=2 * A), EINVAL), (dict(out=5 * A), EINVAL), (dict(k=1 << 18), EUNSUPPORTED),
    (dict(m=1 << 24, n=1 << 21, out_stride=1 << 21), EUNSUPPORTED),
])
def test_matmul_refuses(bad, status):
    assert matmul(**bad) == status


def test_without_rows_needs_no_device():
    assert quantize(rows=0) == OK and matmul(m=0) == OK


def rotary(tensors=None, count=None, plan=None, cells=None, table=A, batch=2, tokens=40, **over):
    a = dict(T=2, H=4, W=5, head_dim=64, dim=(16, 24, 24), type=BF16, theta=1e4, origin=(0, 0, 0), step=(1, 1, 1), flags=0, reserved=0)
    a.update(over)
    cfg = J.jenga_rotary_config(a["T"], a["H"], a["W"], a["head_dim"], (ctypes.c_int32 * 3)(*a["dim"]), a["type"], a["theta"],
                                (ctypes.c_double * 3)(*a["origin"]), (ctypes.c_double * 3)(*a["step"]), a["flags"], a["reserved"])
    tensors = tensors or [dict()]
    list_ = (J.jenga_rotary_tensor * 2)()
    for i, (t, o) in enumerate(zip(list_, tensors)):
        d = dict(src=(4 + 16 * i) * A, dst=(12 + 16 * i) * A, src_batch=40 * 192, src_token=192, src_head=64, dst_batch=40 * 192, dst_token=192,
                 dst_head=64, heads=3, reserved=0)
        d.update(o)
        for n, v in d.items():
            setattr(t, n, v)
    return J.raw().jenga_rotary(ctypes.byref(cfg), plan, cells, table, list_, count if count is not None else len(tensors), batch, tokens,
                                None)


@pytest.mark.parametrize("bad,status", [
    (dict(T=0), EINVAL), (dict(H=-1), EINVAL), (dict(head_dim=0), EINVAL), (dict(head_dim=65), EUNSUPPORTED),
    (dict(head_dim=2048), EUNSUPPORTED), (dict(dim=(16, 24, 26)), EINVAL), (dict(dim=(0, 0, 0)), EINVAL), (dict(dim=(15, 24, 24)), EINVAL), (dict(dim=(-2, 24, 24)), EINVAL),
    (dict(type=E4M3), EINVAL), (dict(theta=0.0), EINVAL), (dict(theta=NAN), EINVAL), (dict(theta=INF), EINVAL),
    (dict(origin=(0, NAN, 0)), EINVAL), (dict(step=(0, 0, INF)), EINVAL), (dict(flags=4), EINVAL), (dict(reserved=1), EINVAL),
    (dict(T=1 << 12, H=1 << 12, W=2), EUNSUPPORTED), (dict(T=1 << 30, H=1 << 30, W=1 << 30), EUNSUPPORTED),
    (dict(table=None), EINVAL), (dict(table=A + 4), EINVAL), (dict(count=0), EINVAL), (dict(count=3), EINVAL), (dict(batch=-1), EINVAL),
    (dict(tokens=-1), EINVAL), (dict(cells=2 * A + 2), EINVAL), (dict(batch=1 << 20, tokens=1 << 20), EUNSUPPORTED),
    (dict(tensors=[dict(src=None)]), EINVAL), (dict(tensors=[dict(dst=None)]), EINVAL), (dict(tensors=[dict(heads=0)]), EINVAL),
    (dict(tensors=[dict(reserved=1)]), EINVAL), (dict(tensors=[dict(src=4 * A + 1)]), EINVAL), (dict(tensors=[dict(src_head=-1)]), EINVAL),
    (dict(tensors=[dict(dst_head=63)]), EINVAL), (dict(tensors=[dict(dst_token=191)]), EINVAL), (dict(tensors=[dict(dst_batch=0)]), EINVAL),
    (dict(tensors=[dict(dst_token=0)]), EINVAL), (dict(tensors=[dict(dst=4 * A + 2)]), EINVAL),
    (dict(tensors=[dict(dst=4 * A, dst_token=200, dst_batch=8000)]), EINVAL),   # the same address, other strides
    (dict(tensors=[dict(), dict(dst=12 * A + 64)]), EINVAL), (dict(tensors=[dict(), dict(dst=4 * A)]), EINVAL),
    (dict(tensors=[dict(), dict(src=12 * A)]), EINVAL), (dict(tensors=[dict(dst=A)]), EINVAL), (dict(cells=12 * A), EINVAL),
])
def test_rotary_refuses(bad, status):
    assert rotary(**bad) == status


def test_rotary_without_tokens_needs_no_device():
    assert rotary(tokens=0) == OK and rotary(batch=0) == OK


def test_rotary_table_values():
    grid, dims, theta, origin, step = (3, 4, 5), (4, 2, 6), 256.0, (1.0e6, -2.0, 0.25), (1.0, 0.5, 3.0)
    cfg = J.make_rotary(*grid, 16, dims, theta, origin, step)
    got = np.zeros(3 * 4 + 4 * 2 + 5 * 6, dtype=np.float32)
    J.jenga_rotary_table(cfg, got)
    want = []
    for a in range(3):
        for n in range(grid[a]):
            for i in range(dims[a] // 2):
                angle = (origin[a] + step[a] * n) * theta ** (-2.0 * i / dims[a])
                want += [math.cos(angle), math.sin(angle)]
    # an angle of 10^6 is a float64 to 2^-34; the result is rounded once to float32
    assert np.abs(got - np.array(want)).max() <= 2.0 ** -25 + 2.0 ** -32
    assert np.array_equal(got[:2], np.array([math.cos(1e6), math.sin(1e6)], dtype=np.float32))
    for bad in (np.zeros(got.size + 1, np.float32), np.zeros(got.size, np.float64), np.zeros((2 * got.size,), np.float32)[::2]):
        with pytest.raises(J.JengaError):
            J.jenga_rotary_table(cfg, bad)
    assert J.raw().jenga_rotary_table(None, None) == EINVAL


# What the binding looks at itself: shapes, types and strides of torch tensors.
def test_the_binding_refuses():
    def refused(f, *args, **kw):
        with pytest.raises(J.JengaError) as e:
            f(*args, **kw)
        assert e.value.status == EINVAL

    x, y = torch.zeros(4, 64), torch.zeros(4, 64)
    refused(J.jenga_layer_norm, x, y)                                            # on the CPU
    refused(J.jenga_layer_norm, x, torch.zeros(4, 65))
    refused(J.jenga_layer_norm, x.t(), y.t())
    refused(J.jenga_layer_norm, x.double(), y.double())
    refused(J.jenga_layer_norm, x, y, torch.zeros(63))
    refused(J.jenga_layer_norm, x, y, torch.zeros(2, 64))
    refused(J.jenga_layer_norm, x, y, torch.zeros(64), torch.zeros(64, dtype=torch.bfloat16))
    refused(J.jenga_layer_norm, x, torch.zeros(4, 64, dtype=torch.uint8))
    refused(J.jenga_layer_norm, x, y, mean=torch.zeros(3))
    refused(J.jenga_layer_norm, x, y, group_rows=-1)
    refused(J.jenga_layer_norm_grad, x, y, torch.zeros(4, 64), None, None, None)
    refused(J.jenga_layer_norm_grad, x, y, torch.zeros(4, 80)[:, :64], None, torch.zeros(4), torch.zeros(4))
    refused(J.jenga_layer_norm_grad, x, y, torch.zeros(4, 64), None, torch.zeros(4), torch.zeros(4), torch.zeros(2, 64))
    q, s = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    refused(J.jenga_quantize, x, q, s)
    refused(J.jenga_quantize, x, q[:, :64], s)
    refused(J.jenga_quantize, x, q, s, 128)
    refused(J.jenga_quantize, x, q, s, 2)
    refused(J.jenga_matmul, q, s, q, s, torch.zeros(4, 4))                        # four rows of scales for b
    refused(J.jenga_matmul, q, s, q, s[:1], torch.zeros(4, 5))
    refused(J.jenga_matmul, q, s, q, s[:1], torch.zeros(4, 4), torch.zeros(4, dtype=torch.bfloat16))
    cfg, table = J.make_rotary(1, 2, 2, 8, (2, 2, 4)), torch.zeros(2 + 4 + 8)
    h = torch.zeros(1, 4, 2, 8, dtype=torch.bfloat16)
    refused(J.jenga_rotary, cfg, table, h, h)                                    # on the CPU
    refused(J.jenga_rotary, cfg, table[:-1], h, h)
    refused(J.jenga_rotary, cfg, table, h, h.float())
    refused(J.jenga_rotary, cfg, table, h[..., :4], h[..., :4])
    refused(J.jenga_rotary, cfg, table, h, h, cells=torch.zeros(4, 3, dtype=torch.int32))


def test_the_binding_refuses_missing_and_flat_tensors():
    cfg, table = J.make_rotary(1, 2, 2, 8, (2, 2, 4)), torch.zeros(2 + 4 + 8)
    h, q, s = torch.zeros(1, 4, 2, 8, dtype=torch.bfloat16), torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    for call in (lambda: J.jenga_rotary(cfg, table, h, h, k=h), lambda: J.jenga_rotary(cfg, table, h, h, k_out=h),
                 lambda: J.jenga_matmul(q.view(2, 2, 128), s, q, s[:1], torch.zeros(4, 4)),
                 lambda: J.jenga_matmul(q, s, q.view(-1), s[:1], torch.zeros(4, 4)),
                 lambda: J.jenga_forward_rotary(None, cfg, table, h[0], h[0], h[0], *[None] * 13)):
        with pytest.raises(J.JengaError) as e:
            call()
        assert e.value.status == EINVAL


@pytest.mark.parametrize("bad", [dict(step=(1e308, 1.0, 1.0)), dict(theta=1e-300, origin=(0.0, 0.0, 1e150))])
def test_rotary_table_refuses_angles_that_are_not_finite(bad):
    cfg = J.make_rotary(3, 4, 5, 16, (4, 2, 6), **bad)
    with pytest.raises(J.JengaError) as e:
        J.jenga_rotary_table(cfg, np.zeros(3 * 4 + 4 * 2 + 5 * 6, dtype=np.float32))
    assert e.value.status == EINVAL


def test_the_binding_refuses_numbers_that_do_not_fit():
    x, y = torch.zeros(4, 64), torch.zeros(4, 64)
    for call in (lambda: J.jenga_layer_norm(x, y, eps=1e300), lambda: J.jenga_layer_norm(x, y, weight_offset=-1e300),
                 lambda: J.jenga_layer_norm(x, y, group_rows=1 << 70)):
        with pytest.raises(J.JengaError) as e:
            call()
        assert e.value.status == EINVAL
