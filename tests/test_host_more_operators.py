"""CPU tests of the norm without a mean, the 4-bit products and dense attention: what they refuse, before any device is touched, sizes of
workspaces, what the binding makes of torch tensors."""
import ctypes

import pytest
import torch

import paper_2505_16864_amd as J
from paper_2505_16864_amd import binding as B

BF16, F16, F32, E4M3, E2M1 = range(5)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -3
A = 1 << 20          # addresses that no call gets to read: every call here is refused, or has nothing to do
NAN, INF = float("nan"), float("inf")


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(J.jenga_rms_config) == 104 and J.jenga_rms_config.heads.offset == 72 and J.jenga_rms_config.eps.offset == 92
    assert ctypes.sizeof(J.jenga_dense_config) == 112 and J.jenga_dense_config.sequences.offset == 80 and J.jenga_dense_config.scale.offset == 104
    assert B._RMS.size == 104 and B._DENSE.size == 112


def rms(call="forward", **over):
    a = dict(rows=4, x_row=64, x_head=64, add_row=64, add_head=64, sum_row=64, sum_head=64, y_row=64, y_head=64, heads=1, cols=64, x_type=BF16,
             y_type=BF16, param_type=BF16, eps=1e-6, weight_offset=0.0, reserved=0, x=A, add=2 * A, weight=3 * A, total=4 * A, y=5 * A, y_scale=None,
             rstd=6 * A, dy=5 * A, dx=4 * A, dweight=8 * A, ws=16 * A, ws_bytes=1 << 40)
    a.update(over)
    cfg = J.jenga_rms_config(*[a[n] for n, _ in J.jenga_rms_config._fields_])
    if call == "forward":
        return J.raw().jenga_rms_norm(ctypes.byref(cfg), a["x"], a["add"], a["weight"], a["total"], a["y"], a["y_scale"], a["rstd"], None)
    return J.raw().jenga_rms_norm_grad(ctypes.byref(cfg), a["x"], a["dy"], a["weight"], a["rstd"], a["add"], a["dx"], a["dweight"], a["ws"],
                                       a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(heads=0), EINVAL), (dict(x_type=E4M3), EINVAL), (dict(x_type=9), EINVAL),
    (dict(y_type=5), EINVAL), (dict(param_type=E2M1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=NAN), EINVAL), (dict(weight_offset=INF), EINVAL),
    (dict(reserved=1), EINVAL), (dict(x_row=-1), EINVAL), (dict(y_head=-1), EINVAL), (dict(add_row=-5), EINVAL), (dict(sum_row=-5), EINVAL),
    (dict(y_type=F32), EUNSUPPORTED), (dict(param_type=F16), EUNSUPPORTED), (dict(cols=1 << 18), EUNSUPPORTED), (dict(rows=1 << 41), EUNSUPPORTED),
    (dict(heads=2, rows=1 << 30), EUNSUPPORTED), (dict(heads=(1 << 20) + 1), EUNSUPPORTED), (dict(x_row=1 << 41), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(x=A + 1), EINVAL), (dict(add=2 * A + 1), EINVAL), (dict(weight=3 * A + 1), EINVAL), (dict(rstd=6 * A + 2), EINVAL),
])
def test_rms_refuses(bad, status):
    assert rms(**bad) == status and rms("grad", **bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(y=None), EINVAL), (dict(y_scale=9 * A), EINVAL), (dict(y_type=E4M3), EINVAL), (dict(y_type=E2M1), EINVAL),
    (dict(y_type=E2M1, y_scale=9 * A, y=5 * A + 8), EINVAL), (dict(y_type=E4M3, y_scale=9 * A + 2), EINVAL),
    (dict(y_type=E2M1, y_scale=9 * A, heads=2), EUNSUPPORTED), (dict(y_type=E2M1, y_scale=5 * A), EINVAL), (dict(y_type=E2M1, y_scale=9 * A, y=A), EINVAL),
    (dict(y_type=E4M3, y_scale=9 * A, y=4 * A), EINVAL),
    (dict(y=A + 2), EINVAL), (dict(y=A, y_row=65), EINVAL), (dict(y=4 * A), EINVAL), (dict(y=3 * A), EINVAL), (dict(y=6 * A), EINVAL),
    (dict(total=A, sum_row=70), EINVAL), (dict(total=2 * A + 4), EINVAL), (dict(total=6 * A), EINVAL), (dict(rstd=A), EINVAL), (dict(rstd=3 * A), EINVAL),
    (dict(y_row=60), EINVAL), (dict(sum_row=0), EINVAL), (dict(heads=3, y_row=192, y_head=63), EINVAL),
])
def test_rms_forward_refuses(bad, status):
    assert rms(**bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(rstd=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=16 * A + 8), EINVAL),
    (dict(ws_bytes=1024 * 64 * 4 - 1), EWORKSPACE), (dict(y_type=E4M3), EUNSUPPORTED), (dict(dx=A), EINVAL), (dict(dx=5 * A), EINVAL),
    (dict(dx=2 * A + 2), EINVAL), (dict(dx=2 * A, sum_row=65), EINVAL), (dict(dweight=4 * A), EINVAL), (dict(dweight=16 * A + 64), EINVAL),
    (dict(dweight=3 * A), EINVAL), (dict(dweight=8 * A + 1), EINVAL), (dict(ws=2 * A), EINVAL), (dict(sum_row=0), EINVAL),
])
def test_rms_gradient_refuses(bad, status):
    assert rms("grad", **bad) == status


# In place, columns of one matrix, an input that is the same for all rows: taken.  (A workspace that is too small is looked at last.)
def test_rms_takes():
    few = dict(ws_bytes=0)
    assert rms("grad", dx=2 * A, **few) == EWORKSPACE                                           # over dtotal
    assert rms("grad", dx=A + 2 * 70, x_row=200, sum_row=200, add=None, **few) == EWORKSPACE    # between the rows of x
    assert rms("grad", y_row=0, **few) == EWORKSPACE                                            # dy of a sum
    assert rms("grad", heads=3, x_row=576, x_head=64, dx=A + 2 * 192, sum_row=576, add=None, y_row=192, **few) == EWORKSPACE
    assert rms(rows=0) == OK and rms("grad", rows=0) == OK
    assert J.jenga_rms_norm_grad_workspace(100, 64) == 1024 * 64 * 4
    with pytest.raises(J.JengaError) as e:
        J.jenga_rms_norm_grad_workspace(100, 1 << 18)
    assert e.value.status == EUNSUPPORTED


def quantize(**over):
    a = dict(x=A, x_stride=64, x_type=BF16, rows=4, cols=64, q=2 * A, scale=3 * A)
    a.update(over)
    return J.raw().jenga_quantize_mx(a["x"], a["x_stride"], a["x_type"], a["rows"], a["cols"], a["q"], a["scale"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(scale=None), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL),
    (dict(x_stride=63), EINVAL), (dict(x_type=E4M3), EINVAL), (dict(x=A + 1), EINVAL), (dict(q=2 * A + 8), EINVAL), (dict(scale=3 * A + 2), EINVAL),
    (dict(q=A), EINVAL), (dict(scale=2 * A + 16), EINVAL), (dict(scale=A + 8), EINVAL), (dict(cols=1 << 18, x_stride=1 << 18), EUNSUPPORTED),
    (dict(rows=(1 << 30) + 1), EUNSUPPORTED), (dict(rows=0), OK),
])
def test_quantize_refuses(bad, status):
    assert quantize(**bad) == status


def matmul(**over):
    a = dict(m=4, out_stride=64, n=64, k=256, out_type=BF16, reserved=0, a=A, a_scale=2 * A, b=3 * A, b_scale=4 * A, bias=5 * A, out=6 * A)
    a.update(over)
    cfg = J.jenga_matmul_config(*[a[n] for n, _ in J.jenga_matmul_config._fields_])
    return J.raw().jenga_matmul_mx(ctypes.byref(cfg), a["a"], a["a_scale"], a["b"], a["b_scale"], a["bias"], a["out"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(a=None), EINVAL), (dict(a_scale=None), EINVAL), (dict(b=None), EINVAL), (dict(b_scale=None), EINVAL), (dict(out=None), EINVAL),
    (dict(m=-1), EINVAL), (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(k=200), EINVAL), (dict(out_stride=63), EINVAL), (dict(reserved=1), EINVAL),
    (dict(out_type=E2M1), EINVAL), (dict(a=A + 8), EINVAL), (dict(b=3 * A + 1), EINVAL), (dict(a_scale=2 * A + 2), EINVAL), (dict(bias=5 * A + 2), EINVAL),
    (dict(out=6 * A + 1), EINVAL), (dict(out=A), EINVAL), (dict(out=3 * A + 16), EINVAL), (dict(out=2 * A), EINVAL), (dict(out=4 * A + 8), EINVAL),
    (dict(out=5 * A), EINVAL), (dict(k=1 << 18), EUNSUPPORTED), (dict(m=1 << 24, n=1 << 21, out_stride=1 << 21), EUNSUPPORTED), (dict(m=0), OK),
])
def test_matmul_refuses(bad, status):
    assert matmul(**bad) == status


def dense(**over):
    a = dict(q_rows=40, kv_rows=50, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, out_row=256, out_head=64, sequences=3, heads=4,
             kv_heads=2, head_dim=64, type=BF16, flags=1, scale=0.125, reserved=0, q=A, k=2 * A, v=3 * A, q_start=4 * A, kv_start=5 * A, kv_len=None,
             out=6 * A, ws=16 * A, ws_bytes=0)
    a.update(over)
    cfg = J.jenga_dense_config(*[a[n] for n, _ in J.jenga_dense_config._fields_])
    return J.raw().jenga_dense_attn(ctypes.byref(cfg), a["q"], a["k"], a["v"], a["q_start"], a["kv_start"], a["kv_len"], a["out"], a["ws"],
                                    a["ws_bytes"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(), EWORKSPACE), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL), (dict(q_start=None), EINVAL),
    (dict(kv_start=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=16 * A + 128), EINVAL), (dict(q_rows=-1), EINVAL), (dict(kv_rows=-1), EINVAL),
    (dict(sequences=-1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(kv_heads=3), EINVAL), (dict(head_dim=0), EINVAL),
    (dict(type=F32), EINVAL), (dict(flags=2), EINVAL), (dict(scale=NAN), EINVAL), (dict(scale=INF), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=-0.1), EINVAL), (dict(scale=1e-40), EINVAL), (dict(reserved=1), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(sequences=1 << 17), EUNSUPPORTED),
    (dict(heads=1 << 13), EUNSUPPORTED), (dict(q_rows=1 << 31), EUNSUPPORTED), (dict(kv_rows=1 << 31), EUNSUPPORTED), (dict(k_row=1 << 24), EUNSUPPORTED),
    (dict(q_row=-1), EINVAL), (dict(v_head=-1), EINVAL), (dict(q=A + 1), EINVAL), (dict(q_start=4 * A + 2), EINVAL), (dict(kv_len=7 * A + 1), EINVAL),
    (dict(out=2 * A), EINVAL), (dict(out=3 * A + 100), EINVAL), (dict(out=A + 2), EINVAL), (dict(out=A, out_row=260), EINVAL), (dict(out=4 * A), EINVAL),
    (dict(out=16 * A), EINVAL), (dict(ws=2 * A), EINVAL), (dict(ws=4 * A), EINVAL), (dict(out_row=128), EINVAL), (dict(out_head=0), EINVAL),
    (dict(out=A), EWORKSPACE), (dict(kv_rows=0), EWORKSPACE), (dict(k=2 * A, v=2 * A), EWORKSPACE), (dict(q_row=0), EWORKSPACE),
    (dict(k=A + 2 * 256, q_row=512, k_row=512), EWORKSPACE), (dict(q_rows=0, ws_bytes=1 << 30), OK), (dict(sequences=0, ws_bytes=1 << 30), OK),
    (dict(q_rows=1 << 30, heads=64, kv_heads=64, q_row=4096, out_row=4096), EUNSUPPORTED),
])
def test_dense_refuses(bad, status):
    assert dense(**bad) == status


def test_dense_workspace():
    few, many = J.jenga_dense_attn_workspace(16, 50000, 16, 40, 8, 128), J.jenga_dense_attn_workspace(60000, 60000, 9, 40, 8, 128)
    assert 1 << 20 < few < 64 << 20          # results of parts, 8 KiB each
    assert many < 1 << 20                    # nothing is cut
    with pytest.raises(J.JengaError) as e:
        J.jenga_dense_attn_workspace(16, 16, 1, 4, 4, 80)
    assert e.value.status == EUNSUPPORTED


# ---- the binding

class _OnGpu(torch.Tensor):
    """A CPU tensor that says it is on GPU 0: what is launched is looked at, and nothing is."""

    def get_device(self):
        return 0


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


def _calls():
    u8, bf, i32 = torch.uint8, torch.bfloat16, torch.int32
    x, y, stats, q, s = _t(4, 64), _t(4, 64), _t(4), _t(4, 64, dtype=u8), _t(4, 4, dtype=u8)
    h, start, room = _t(4, 2, 64, dtype=bf), _t(3, dtype=i32), _t(512, dtype=u8)
    return {"quantize_mx": lambda **kw: J.jenga_quantize_mx(x, q, s, **kw),
            "matmul_mx": lambda **kw: J.jenga_matmul_mx(q, s, q, s, _t(4, 4), **kw),
            "rms_norm": lambda **kw: J.jenga_rms_norm(x, y, **kw),
            "rms_norm_grad": lambda **kw: J.jenga_rms_norm_grad(x, y, _t(4, 64), None, stats, **kw),
            "dense_attn": lambda **kw: J.jenga_dense_attn(h, h, h, _t(4, 2, 64, dtype=bf), start, start, workspace=room, **kw)}


class _Recorder:
    def __init__(self):
        self.seen = []

    def jenga_strerror(self, status):
        return b""

    def __getattr__(self, call):
        return lambda *args: self.seen.append((call, args)) or 0


@pytest.fixture
def recorder(monkeypatch):
    r = _Recorder()
    B._use_torch()
    monkeypatch.setattr(B, "_lib", r)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_current_stream", lambda device: 1000 + device, raising=False)
    return r


@pytest.mark.parametrize("name", ["quantize_mx", "matmul_mx", "rms_norm", "rms_norm_grad", "dense_attn"])
def test_calls_go_to_the_current_stream(name, recorder):
    call = _calls()[name]
    call()
    call(stream=77)
    call(stream=0)
    assert [(c, a[-1]) for c, a in recorder.seen] == [("jenga_" + name, 1000), ("jenga_" + name, 77), ("jenga_" + name, 0)]


def _refused(f):
    with pytest.raises(J.JengaError) as e:
        f()
    assert e.value.status == -1


# Before the first call of a process the types are not there yet.
def test_tensors_of_other_devices_are_refused(monkeypatch):
    B._use_torch()
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    for call in _calls().values():
        _refused(call)
    cpu = torch.zeros(4, 64)
    _refused(lambda: J.jenga_rms_norm(cpu, cpu.clone()))
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    x = _t(4, 64)
    for kw in (dict(weight=torch.zeros(64)), dict(residual=torch.zeros(4, 64)), dict(total=torch.zeros(4, 64)), dict(rstd=torch.zeros(4))):
        _refused(lambda: J.jenga_rms_norm(x, _t(4, 64), **kw))


def test_shapes_and_types_are_refused(recorder):
    x, y, u8, bf = _t(4, 64), _t(4, 64), torch.uint8, torch.bfloat16
    bad = [lambda: J.jenga_rms_norm(x, _t(4, 63)), lambda: J.jenga_rms_norm(x, _t(4, 64, dtype=bf)), lambda: J.jenga_rms_norm(_t(64), _t(64)),
           lambda: J.jenga_rms_norm(x, y, weight=_t(4, 64)), lambda: J.jenga_rms_norm(x, y, weight=_t(128)[::2]),
           lambda: J.jenga_rms_norm(x, y, residual=_t(3, 64)), lambda: J.jenga_rms_norm(x, y, rstd=_t(4, 1)),
           lambda: J.jenga_rms_norm(x, _t(4, 64, dtype=u8)), lambda: J.jenga_rms_norm(x, _t(4, 64, dtype=u8), y_scale=_t(4, 3, dtype=u8)),
           lambda: J.jenga_rms_norm(x, y, y_scale=_t(4, 4, dtype=u8)), lambda: J.jenga_rms_norm(_t(4, 128)[:, ::2], y),
           lambda: J.jenga_rms_norm(_t(4, 2, 64), _t(4, 64, dtype=u8), y_scale=_t(4, 4, dtype=u8)),
           lambda: J.jenga_rms_norm_grad(x, y, _t(4, 64), None, None), lambda: J.jenga_rms_norm_grad(x, y, _t(4, 64), None, _t(4), dweight=_t(1, 64)),
           lambda: J.jenga_quantize_mx(x, _t(4, 128, dtype=u8), _t(4, 4, dtype=u8)), lambda: J.jenga_quantize_mx(x, _t(4, 64, dtype=u8), _t(4, 2, dtype=u8)),
           lambda: J.jenga_quantize_mx(_t(64), _t(4, 64, dtype=u8), _t(4, 4, dtype=u8)),
           lambda: J.jenga_matmul_mx(_t(4, 64, dtype=u8), _t(4, 4, dtype=u8), _t(3, 128, dtype=u8), _t(3, 8, dtype=u8), _t(4, 3)),
           lambda: J.jenga_matmul_mx(_t(4, 64, dtype=u8), _t(4, 4, dtype=u8), _t(3, 64, dtype=u8), _t(3, 4, dtype=u8), _t(4, 4)),
           lambda: J.jenga_matmul_mx(_t(4, 64, dtype=u8), _t(4, 4, dtype=u8), _t(3, 64, dtype=u8), _t(3, 4, dtype=u8), _t(4, 3), _t(4))]
    h, start, room = _t(4, 2, 64, dtype=bf), _t(3, dtype=torch.int32), _t(512, dtype=u8)
    bad += [lambda: J.jenga_dense_attn(h, h, h, h[:3], start, start, workspace=room), lambda: J.jenga_dense_attn(h, h, _t(5, 2, 64, dtype=bf), h, start, start, workspace=room),
            lambda: J.jenga_dense_attn(h, h, h, _t(4, 2, 64), start, start, workspace=room), lambda: J.jenga_dense_attn(h, h, h, h, start, start[:2], workspace=room),
            lambda: J.jenga_dense_attn(h, h, h, h, start.long(), start, workspace=room), lambda: J.jenga_dense_attn(h, h, h, h, start, start),
            lambda: J.jenga_dense_attn(h, h, h, h, start, start, kv_len=start, workspace=room), lambda: J.jenga_dense_attn(h[:, 0], h, h, h, start, start, workspace=room),
            lambda: J.jenga_dense_attn(h, _t(4, 2, 32, dtype=bf), h, h, start, start, workspace=room)]
    for f in bad:
        _refused(f)
    assert recorder.seen == []


def test_sizes_and_strides_of_tensors(recorder):
    qkv = _t(5, 3, 4, 64)
    J.jenga_rms_norm(qkv[:, 1], qkv[:, 1], _t(64))
    cfg = dict(zip((n for n, _ in J.jenga_rms_config._fields_), B._RMS.unpack(recorder.seen[-1][1][0])))
    assert (cfg["rows"], cfg["heads"], cfg["cols"], cfg["x_row"], cfg["x_head"], cfg["y_row"], cfg["y_head"]) == (5, 4, 64, 768, 64, 768, 64)
    for dtype, kind in ((torch.uint8, E2M1), (torch.float8_e4m3fn, E4M3)):
        J.jenga_rms_norm(_t(5, 100), _t(5, 64 if kind == E2M1 else 128, dtype=torch.uint8).view(dtype), y_scale=_t(5, 4, dtype=torch.uint8))
        cfg = dict(zip((n for n, _ in J.jenga_rms_config._fields_), B._RMS.unpack(recorder.seen[-1][1][0])))
        assert (cfg["x_type"], cfg["y_type"], cfg["heads"]) == (F32, kind, 1)
    h = _t(2, 7, 64, dtype=torch.float16).transpose(0, 1)
    J.jenga_dense_attn(h, _t(0, 2, 64, dtype=torch.float16), _t(0, 2, 64, dtype=torch.float16), _t(7, 2, 64, dtype=torch.float16),
                       _t(2, dtype=torch.int32), _t(2, dtype=torch.int32), causal=True, workspace=_t(256, dtype=torch.uint8))
    cfg = dict(zip((n for n, _ in J.jenga_dense_config._fields_), B._DENSE.unpack(recorder.seen[-1][1][0])))
    assert (cfg["q_row"], cfg["q_head"], cfg["out_row"], cfg["kv_rows"], cfg["type"], cfg["flags"], cfg["scale"]) == (64, 448, 128, 0, F16, 1, 0.125)
    assert all(p for p in recorder.seen[-1][1][1:6])      # addresses though there are no keys
    count = len(recorder.seen)
    for f in (lambda: J.jenga_rms_norm(_t(0, 64), _t(0, 64)), lambda: J.jenga_quantize_mx(_t(0, 64), _t(0, 64, dtype=torch.uint8), _t(0, 4, dtype=torch.uint8))):
        f()
    assert len(recorder.seen) == count
