"""jenga_dense_attn over keys that are cut into many parts: what joins them takes every one.  Values have an offset, so that a part that is left out shows:
it takes a 64th of the offset at least with it, 0.06 of 4, where 0.04 of it is the tolerance (bf16: half a step of probabilities and one of results)."""
import pytest
import torch

from more_operator_util import attention
from operator_util import TYPES, check, randn

pytestmark = pytest.mark.gpu


def _compare(q_lens, kv_lens, heads, kv_heads, d, dtype, seed, causal=True):
    import paper_2505_16864_amd as J
    t = TYPES[dtype]
    q, k = randn(seed, sum(q_lens), heads, d).to(t), randn(seed + 1, sum(kv_lens), kv_heads, d).to(t)
    v = (randn(seed + 2, sum(kv_lens), kv_heads, d) / 4 + 4).to(t)
    starts = [[0] + torch.tensor(n).cumsum(0).tolist() for n in (q_lens, kv_lens)]
    want, tol = attention(q, k, v, q_lens, list(zip(starts[1], kv_lens)), causal, d ** -0.5, t)
    q_start, kv_start = [torch.tensor(s, dtype=torch.int32, device="cuda:0") for s in starts]
    size = J.jenga_dense_attn_workspace(sum(q_lens), sum(kv_lens), len(q_lens), heads, kv_heads, d)
    room = torch.full((size,), 255, dtype=torch.uint8, device="cuda:0")       # NaN, if any of it were read before it is written
    out = torch.full(q.shape, 9.0, dtype=t, device="cuda:0")
    J.jenga_dense_attn(q.cuda(), k.cuda(), v.cuda(), out, q_start, kv_start, causal=causal, workspace=room)
    torch.cuda.synchronize()
    check(out, want, tol)


# A part is 256 keys at least: 17 to 64 parts of one token's keys, the last parts in turn in every group of lanes.
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128)])
@pytest.mark.parametrize("keys", [4097, 4352, 4700, 8193, 8448, 8500, 8700, 9000, 10300, 12300, 12545, 12700, 13000, 14400, 16300, 16500, 20000])
def test_one_token_over_many_parts(keys, dtype, d):
    _compare([1], [keys], 2, 1, d, dtype, keys)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [8300, 4200]), ([2, 1, 1], [4353, 10300, 700]), ([4], [12400]), ([1, 0, 1], [16400, 40, 9])])
def test_sequences_of_different_parts(q_lens, kv_lens, d):
    _compare(q_lens, kv_lens, 5, 1, d, "bf16", 3)


# More sequences than a wavefront looks at: the list.
@pytest.mark.parametrize("keys", [4300, 8400])
@pytest.mark.parametrize("d", [64, 128])
def test_parts_of_a_list(keys, d):
    _compare([1] * 70, [20] * 30 + [keys] + [11] * 38 + [4300], 2, 1, d, "bf16", 5)


# Tiles of 128 rows, whose parts are joined elsewhere.
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("keys", [8300, 16500])
def test_prompts_over_many_parts(keys, causal):
    _compare([70], [keys], 1, 1, 64, "bf16", 7, causal)
