"""CPU test of the binding: a workspace is memory without gaps or repeats, so that its elements are the bytes that the call may write."""
import pytest
import torch

import paper_2505_16864_amd as J
from paper_2505_16864_amd import binding as B


class _OnGpu(torch.Tensor):
    """A CPU tensor that says it is on GPU 0: what is launched is looked at, and nothing is."""

    def get_device(self):
        return 0


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


class _Recorder:
    def __init__(self):
        self.seen = []

    def jenga_strerror(self, status):
        return b""

    def __getattr__(self, call):
        return lambda *args: self.seen.append(args) or 0


CALLS = {
    "dense_attn": lambda room: J.jenga_dense_attn(*[_t(4, 2, 64, dtype=torch.bfloat16) for _ in range(4)], *[_t(3, dtype=torch.int32) for _ in range(2)],
                                                  workspace=room),
    "rms_norm_grad": lambda room: J.jenga_rms_norm_grad(*[_t(4, 64) for _ in range(3)], None, _t(4), dweight=_t(64), workspace=room),
    "layer_norm_grad": lambda room: J.jenga_layer_norm_grad(*[_t(4, 64) for _ in range(3)], _t(1, 64), _t(4), _t(4), dweight=_t(1, 64), workspace=room),
}


@pytest.mark.parametrize("name", CALLS)
def test_workspaces(name, monkeypatch):
    r = _Recorder()
    B._use_torch()
    monkeypatch.setattr(B, "_lib", r)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_current_stream", lambda device: 1000 + device)
    for room in (_t(1, 256).expand(4096, 256), _t(64, 64)[:, :32], _t(4096)[::2]):
        with pytest.raises(J.JengaError) as e:
            CALLS[name](room)
        assert e.value.status == -1
    assert r.seen == []
    for room, size in ((_t(16, 64), 4096), (_t(1000, dtype=torch.uint8), 1000), (_t(64, 64)[8:16], 2048)):
        CALLS[name](room)
        assert r.seen[-1][-2] == size and r.seen[-1][-3] == room.data_ptr()
