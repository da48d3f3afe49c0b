"""jenga_dense_attn where the last tile of a sequence begins inside its last token: rows of it that are not there have nothing to do with the token's other
heads, which belong to another tile."""
import pytest
import torch

from more_operator_util import attention
from operator_util import TYPES, check, randn

pytestmark = pytest.mark.gpu

# tokens, heads on one of keys: 20 packed rows in tiles of 16; 130 and 260 in tiles of 128; 40 x 27 = 1080 rows, the last tile at 1024 in token 25, which is not the last
CASES = [(1, 20), (26, 5), (13, 20), (1, 17), (27, 40), (52, 5)]


def _call(q, k, v, out, lens=None):
    import paper_2505_16864_amd as J
    room = torch.empty(J.jenga_dense_attn_workspace(q.shape[0], k.shape[0], 1, q.shape[1], k.shape[1], q.shape[2]), dtype=torch.uint8, device="cuda:0")
    starts = [torch.tensor([0, n], dtype=torch.int32, device="cuda:0") for n in (q.shape[0], k.shape[0])]
    J.jenga_dense_attn(q, k, v, out, *starts, causal=True, workspace=room)
    torch.cuda.synchronize()


def _inputs(tokens, heads, keys, d, dtype):
    t = TYPES[dtype]
    return randn(1, tokens, heads, d).to(t).cuda(), (3 * randn(2, keys, 1, d)).to(t).cuda(), randn(3, keys, 1, d).to(t).cuda()


# The last tile's rows have the same bits whatever the heads of its last token that are in the tile before hold.
@pytest.mark.parametrize("tokens,heads", CASES)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_bits_do_not_follow_another_tiles_rows(tokens, heads, dtype, d):
    q, k, v = _inputs(tokens, heads, 900, d, dtype)
    tile = 16 if tokens <= 4 and tokens * heads <= 32 else 128
    first = tokens * heads // tile * tile                       # the last tile's first row
    want = torch.empty_like(q)
    _call(q, k, v, want)
    for bad in (float("nan"), 100.0):
        other = q.clone()
        other.view(-1, d)[:first] = bad
        got = torch.empty_like(q)
        _call(other, k, v, got)
        assert torch.equal(got.view(-1, d)[first:], want.view(-1, d)[first:]), bad


# Over q: the same bits as into another tensor, every time.
@pytest.mark.parametrize("tokens,heads", CASES)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_over_q(tokens, heads, dtype, d):
    q, k, v = _inputs(tokens, heads, 900, d, dtype)
    apart = torch.empty_like(q)
    _call(q, k, v, apart)
    want, tol = attention(q.cpu(), k.cpu(), v.cpu(), [tokens], [(0, 900)], True, d ** -0.5, q.dtype)
    check(apart, want, tol)
    for _ in range(5):
        over = q.clone()
        _call(over, k, v, over)
        assert torch.equal(over, apart)
