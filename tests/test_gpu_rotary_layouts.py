"""jenga_rotary in place on tensors that lie between each other, down to one token of each sequence, against float64 and by its bits.

Tolerance: cos and sin rounded to float32, two products and a sum: 4 u (|x| + |y|) of the pair, u = 2^-24, and one rounding."""
import pytest
import torch

from operator_util import U32, check, half_step, randn, rotary

pytestmark = pytest.mark.gpu

GRID = (2, 3, 5)


# Columns of one projection [batch, tokens, 3, heads, D] and heads one behind the other [batch, 3, heads, tokens, D].
@pytest.mark.parametrize("by_heads", [False, True])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("head_dim,dims", [(64, (16, 24, 24)), (10, (2, 4, 2))])
@pytest.mark.parametrize("batch,tokens", [(2, 1), (5, 1), (2, 2), (3, 33)])
def test_in_place(batch, tokens, head_dim, dims, halves, by_heads):
    import paper_2505_16864_amd as J
    cfg = J.make_rotary(*GRID, head_dim, dims, origin=(1, 2, 3), flags=J.JENGA_ROTARY_HALVES if halves else 0)
    table = torch.empty(sum(n * d for n, d in zip(GRID, dims)))
    J.jenga_rotary_table(cfg, table)
    heads = 3
    if by_heads:
        data = randn(batch + tokens, batch, 3, heads, tokens, head_dim).to(torch.bfloat16)
        parts = lambda t: [t[:, i].transpose(1, 2) for i in range(3)]  # noqa: E731
    else:
        data = randn(batch + tokens, batch, tokens, 3, heads, head_dim).to(torch.bfloat16)
        parts = lambda t: t.unbind(2)  # noqa: E731
    qkv = data.cuda()
    q, v, k = parts(qkv)
    apart = [torch.empty((batch, tokens, heads, head_dim), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    J.jenga_rotary(cfg, table.cuda(), q, apart[0], k, apart[1])
    J.jenga_rotary(cfg, table.cuda(), q, q, k, k)
    torch.cuda.synchronize()
    assert torch.equal(q, apart[0]) and torch.equal(k, apart[1]) and torch.equal(v.cpu(), parts(data)[1])
    for got, x in ((q, parts(data)[0].double()), (k, parts(data)[2].double())):
        want = rotary(x, *GRID, dims, 10000.0, (1, 2, 3), halves=halves)
        top = x.abs().topk(2, dim=-1).values.sum(-1, keepdim=True)
        check(got, want, half_step(torch.bfloat16) * want.abs() + 4 * U32 * top * 1.01)


# A result that does lie over another tensor, by a part of one head.
@pytest.mark.parametrize("tokens", [1, 2])
def test_refuses_a_shared_part(tokens):
    import paper_2505_16864_amd as J
    cfg, dims = J.make_rotary(*GRID, 64, (16, 24, 24)), (16, 24, 24)
    table = torch.zeros(sum(n * d for n, d in zip(GRID, dims)), device="cuda:0")
    room = torch.zeros((2, tokens, 3 * 3 * 64), dtype=torch.bfloat16, device="cuda:0")
    q, k = [room[:, :, i:i + 192].view(2, tokens, 3, 64) for i in (0, 160)]
    with pytest.raises(J.JengaError) as e:
        J.jenga_rotary(cfg, table, q, q, k, k)
    assert e.value.status == -1
    torch.cuda.synchronize()
    assert not room.any()


# From one layout to another: tokens first to heads first, one head for all (stride 0), one sequence for all, K beside Q with fewer heads.
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("head_dim,dims", [(64, (16, 24, 24)), (10, (2, 4, 2))])
@pytest.mark.parametrize("tokens", [1, 37])
def test_from_one_layout_to_another(tokens, head_dim, dims, halves):
    import paper_2505_16864_amd as J
    cfg = J.make_rotary(*GRID, head_dim, dims, flags=J.JENGA_ROTARY_HALVES if halves else 0)
    table = torch.empty(sum(n * d for n, d in zip(GRID, dims)))
    J.jenga_rotary_table(cfg, table)
    q, k = randn(1, 3, tokens, 1, head_dim).to(torch.bfloat16), randn(2, 1, tokens, 2, head_dim).to(torch.bfloat16)
    q_out, k_out = [torch.full((3, heads, tokens, head_dim), 7.0, dtype=torch.bfloat16, device="cuda:0").transpose(1, 2) for heads in (5, 2)]
    J.jenga_rotary(cfg, table.cuda(), q.cuda().expand(-1, -1, 5, -1), q_out, k.cuda().expand(3, -1, -1, -1), k_out)
    torch.cuda.synchronize()
    for got, x in ((q_out, q.double().expand(-1, -1, 5, -1)), (k_out, k.double().expand(3, -1, -1, -1))):
        want = rotary(x, *GRID, dims, 10000.0, halves=halves)
        top = x.abs().topk(2, dim=-1).values.sum(-1, keepdim=True)
        check(got, want, half_step(torch.bfloat16) * want.abs() + 4 * U32 * top * 1.01)
