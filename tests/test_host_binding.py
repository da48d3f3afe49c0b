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
