"""CPU tests of what the binding makes of torch tensors before a call: sizes, strides, streams."""
import pytest
import torch

import paper_2505_16864_amd as J
from paper_2505_16864_amd import binding as B


def _fields(packed):
    return dict(zip((n for n, _ in B.jenga_norm_config._fields_), B._NORM.unpack(packed)))


# A single row has no distance to a next one: torch calls it contiguous whatever its stride says, and so does jenga_quantize.
@pytest.mark.parametrize("dtype", [torch.uint8, torch.float8_e4m3fn])
def test_one_row_of_8_bits_from_a_wider_tensor(dtype):
    x = torch.zeros(1, 100)
    for y in (torch.zeros(1, 512, dtype=torch.uint8).view(dtype)[:, :128], torch.zeros(3, 384, dtype=torch.uint8).view(dtype)[1:2, 128:256]):
        assert y.is_contiguous() and y.stride(0) > 128
        assert _fields(B._norm_config("call", x, y, None, None, 0, 0.0, 1e-6))["y_stride"] == 128


def test_rows_of_8_bits_lie_next_to_each_other():
    for y in (torch.zeros(2, 512, dtype=torch.uint8)[:, :128], torch.zeros(2, 100, dtype=torch.uint8), torch.zeros(1, 128, dtype=torch.uint8)):
        with pytest.raises(J.JengaError) as e:
            J.jenga_layer_norm(torch.zeros(2, 100), y, y_scale=torch.zeros(2, 4, dtype=torch.uint8))
        assert e.value.status == -1


@pytest.mark.parametrize("shape", [(), (1, 1, 64)])
def test_weights_that_are_no_rows_are_refused(shape):
    x, y = torch.zeros(4, 64), torch.zeros(4, 64)
    for kw in (dict(weight=torch.zeros(shape)), dict(bias=torch.zeros(shape))):
        with pytest.raises(J.JengaError) as e:
            J.jenga_layer_norm(x, y, **kw)
        assert e.value.status == -1


class _OnGpu(torch.Tensor):
    """A CPU tensor that says it is on GPU 0: what is launched is looked at, and nothing is."""

    def get_device(self):
        return 0


def _calls():
    t = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)  # noqa: E731
    u8, bf = torch.uint8, torch.bfloat16
    x, y, stats = t(4, 64), t(4, 64), t(4)
    q, s = t(4, 128, dtype=u8), t(4, 4, dtype=u8)
    cfg, h = J.make_rotary(1, 2, 2, 64, (16, 24, 24)), t(1, 4, 2, 64, dtype=bf)
    table = t(16 + 48 + 48)
    return {"quantize": lambda **kw: J.jenga_quantize(x, q, s, **kw),
            "matmul": lambda **kw: J.jenga_matmul(q, s, q, s[:1], t(4, 4), **kw),
            "layer_norm": lambda **kw: J.jenga_layer_norm(x, y, **kw),
            "layer_norm_grad": lambda **kw: J.jenga_layer_norm_grad(x, y, t(4, 64), None, stats, stats, **kw),
            "rotary": lambda **kw: J.jenga_rotary(cfg, table, h, h, **kw),
            "forward_rotary": lambda **kw: J.jenga_forward_rotary(None, cfg, table, h, h, h, *[None] * 7, 0, None, None, None, 0, None, **kw)}


# Work on tensors that torch's current stream makes or takes away has to be on that stream; another one is the caller's to name.
@pytest.mark.parametrize("name", ["quantize", "matmul", "layer_norm", "layer_norm_grad", "rotary", "forward_rotary"])
def test_calls_on_tensors_go_to_the_current_stream(name, monkeypatch):
    seen = []

    class Recorder:
        def __getattr__(self, call):
            return lambda *args: seen.append((call, args[-1])) or 0

    B._use_torch()
    monkeypatch.setattr(B, "_lib", Recorder())
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_current_stream", lambda device: 1000 + device, raising=False)
    call = _calls()[name]
    call()
    call(stream=77)
    call(stream=0)
    assert seen == [("jenga_" + name, 1000), ("jenga_" + name, 77), ("jenga_" + name, 0)]
