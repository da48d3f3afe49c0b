"""jenga_dense_attn over keys and values whose rows overlap in memory, or are one row for all keys: the step that reaches past the last key finds other keys' values
behind it there, not zeros."""
import pytest
import torch

from more_operator_util import attention
from operator_util import TYPES, check, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("row", [0, 8, 13, 64])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_len,keys", [(1, 40), (3, 33), (1, 5000), (150, 70), (150, 300)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_rows_over_each_other(q_len, keys, causal, row, dtype, d):
    import paper_2505_16864_amd as J
    t = TYPES[dtype]
    q = randn(1, q_len, 2, d).to(t).cuda()
    k = randn(2, keys * 64 + d).to(t).cuda().as_strided((keys, 1, d), (row, d, 1))
    values = randn(3, keys * 64 + d).to(t).cuda()
    # of the first and of the last key: all rows see the first, a causal call's last row the last
    first, last = 5, max(0, keys - 1) * row + d - 3
    values[first], values[last] = float("inf"), float("-inf")
    v = values.as_strided((keys, 1, d), (row, d, 1))
    want, tol = attention(q.cpu(), k.cpu(), v.cpu(), [q_len], [(0, keys)], causal, d ** -0.5, t)
    out = torch.empty_like(q)
    starts = [torch.tensor([0, n], dtype=torch.int32, device="cuda:0") for n in (q_len, keys)]
    room = torch.empty(J.jenga_dense_attn_workspace(q_len, keys, 1, 2, 1, d), dtype=torch.uint8, device="cuda:0")
    J.jenga_dense_attn(q, k, v, out, *starts, causal=causal, workspace=room)
    torch.cuda.synchronize()
    check(out, want, tol)
