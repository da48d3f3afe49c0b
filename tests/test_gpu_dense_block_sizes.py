"""DenseBlock on fewer rows and sequences than it is built for: the results of a block that is built for just these."""
import pytest
import torch

from operator_util import randn
from test_gpu_dense_block import _block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,sequences,lens", [(20000, 8, [60, 1, 139]), (20000, 8, [3000, 2000]), (64, 16, [64]), (64, 16, [40, 3]), (9000, 100, [1] * 70),
                                                 (9000, 100, [8999])])
@pytest.mark.parametrize("heads,kv_heads,d", [(6, 2, 64), (5, 5, 128), (40, 8, 64)])
def test_shorter_batches(rows, sequences, lens, heads, kv_heads, d):
    n, hidden = sum(lens), 192
    starts = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda:0")
    x = randn(1, n, hidden).to(torch.bfloat16).cuda()
    got = []
    for size in ((rows, sequences), (n, len(lens))):
        block, _ = _block(*size, heads, kv_heads, d, hidden, 9, turn=False)
        got.append([t.clone() for t in block.forward(x, starts)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(*got))
