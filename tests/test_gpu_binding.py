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
