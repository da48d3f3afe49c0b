"""The operators together: a carved layer with rotary positions in its re-ordering pass, and a whole block from hidden states to
hidden states, against the single calls, float64 and the oracle."""
import numpy as np
import pytest
import torch

import jenga_inputs as ji
from gpu_util import check_output, oracle_layout, to_f64
from operator_util import U32, check, half_step, held_values, quantize, randn, rotary
from oracle import jenga_oracle as jo

pytestmark = pytest.mark.gpu


def _single_calls(w, dims, theta, flags, q, k, v, **layer):
    """jenga_rotary of Q and K, then jenga_forward."""
    import paper_2505_16864_amd as J
    from paper_2505_16864_amd.layer import CarveLayer
    plain = CarveLayer(w, "cuda:0", want_mask=True, want_lse=True, **layer)
    cfg = J.make_rotary(w["T"], w["H"], w["W"], w["head_dim"], dims, theta, flags=flags)
    table = torch.empty(sum(n * d for n, d in zip((w["T"], w["H"], w["W"]), dims)))
    J.jenga_rotary_table(cfg, table)
    turned = [torch.empty((w["batch"], q.shape[1], w["heads"], w["head_dim"]), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    J.jenga_rotary(cfg, table.cuda(), q, turned[0], k, turned[1])
    out = plain.forward(turned[0], turned[1], v.contiguous())
    torch.cuda.synchronize()
    return plain, out


# Every block size and head size, ragged blocks, several batch entries; Q, K and V apart and as columns of one projection: the same
# bits in every place that a call writes.
@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("block,head_dim,dims", [(32, 64, (16, 24, 24)), (64, 64, (20, 22, 18)), (128, 64, (0, 32, 32)),
                                                 (32, 128, (44, 42, 42)), (64, 128, (16, 56, 56)), (128, 128, (32, 48, 48))])
def test_forward_with_rotary_positions(block, head_dim, dims, halves):
    from paper_2505_16864_amd.layer import CarveLayer
    for grid, n_text, batch in (((3, 9, 11), 37, 2), ((1, 1, 5), 0, 1), ((4, 8, 8), 130, 1)):
        w = dict(T=grid[0], H=grid[1], W=grid[2], n_text=n_text, batch=batch, heads=3, head_dim=head_dim, block=block, topk=0.3, p=0.3)
        qkv = torch.stack(ji.make_qkv(w, 50 + block), dim=2).cuda()          # [batch, tokens, 3, heads, D]
        columns = qkv.unbind(2)
        plain, want = _single_calls(w, dims, 256.0, halves, *columns)
        layer = CarveLayer(w, "cuda:0", want_mask=True, want_lse=True, rotary=dict(dims=dims, theta=256.0, flags=halves))
        for q, k, v in (columns, [t.contiguous() for t in columns]):
            for t in (layer.q_c, layer.k_c, layer.v_c, layer.o_c, layer.out_thw, layer.lse):
                t.fill_(7.0)
            layer.sel_count.fill_(-1)
            got = layer.forward(q, k, v)
            torch.cuda.synchronize()
            for name in ("q_c", "k_c", "v_c", "sel_count", "mask", "o_c", "lse"):
                assert torch.equal(getattr(layer, name), getattr(plain, name)), (grid, name)
            assert torch.equal(got, want), grid


def test_forward_rotary_refuses():
    import paper_2505_16864_amd as J
    from paper_2505_16864_amd.layer import CarveLayer
    w = ji.WORKLOADS["tiny"]
    layer = CarveLayer(w, "cuda:0", rotary=dict(dims=(16, 24, 24)))
    q, k, v = [t.cuda() for t in ji.make_qkv(w, 3)]

    def call(q=q, k=k, v=v, cfg=layer.rotary, **over):
        a = dict(q_c=layer.q_c, k_c=layer.k_c, v_c=layer.v_c, o_c=layer.o_c, out=layer.out_thw, ws=layer.ws_attn, bytes=layer.ws_attn.numel())
        a.update(over)
        J.jenga_forward_rotary(layer.plan, cfg, layer.rotary_table, q, k, v, a["q_c"], a["k_c"], a["v_c"], layer.sel_count, layer.sel_index,
                               None, layer.ws_select, layer.ws_select.numel(), a["o_c"], None, a["ws"], a["bytes"], a["out"])

    call()
    other = J.make_rotary(w["T"], w["H"], w["W"] + 1, w["head_dim"], (16, 24, 24))
    f32 = J.make_rotary(w["T"], w["H"], w["W"], w["head_dim"], (16, 24, 24))
    f32.type = J.JENGA_F32
    for bad, status in ((dict(q_c=q), -1), (dict(q_c=layer.k_c), -1), (dict(out=v), -1), (dict(out=layer.o_c), -1), (dict(o_c=layer.q_c), -1),
                        (dict(bytes=1), -3), (dict(ws=None), -1), (dict(q=q[:, :, :1]), -1), (dict(k=k.float()), -1), (dict(cfg=f32), -1),
                        (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), -1)):
        with pytest.raises(J.JengaError) as e:
            call(**bad)
        assert e.value.status == status, bad
    with pytest.raises(J.JengaError):
        J.jenga_forward_rotary(layer.plan, other, torch.zeros(4 * 16 + 8 * 24 + 9 * 24, device="cuda:0"), q, k, v, layer.q_c, layer.k_c, layer.v_c,
                               layer.sel_count, layer.sel_index, None, layer.ws_select, layer.ws_select.numel(), layer.o_c, None, layer.ws_attn,
                               layer.ws_attn.numel(), layer.out_thw)
    torch.cuda.synchronize()


def _block(w, hidden, seed, dtype=torch.bfloat16, **kw):
    from paper_2505_16864_amd.layer import CarveBlock
    inner = w["heads"] * w["head_dim"]
    w_qkv = randn(seed, 3 * inner, hidden) / hidden ** 0.5
    w_out = randn(seed + 1, hidden, inner) / inner ** 0.5
    b_qkv, b_out = 0.1 * randn(seed + 2, 3 * inner), 0.1 * randn(seed + 3, hidden)
    weights = (w_qkv.to(dtype), b_qkv.float(), w_out.to(dtype), b_out.float())
    d = w["head_dim"]
    return CarveBlock(w, *weights, rotary=dict(dims=(d // 4, d // 4 + 4, d // 2 - 4), theta=256.0), **kw), weights


# The whole block, each stage against float64 from what the stage before it left.
@pytest.mark.parametrize("name,hidden", [("tiny", 200), ("small", 640)])
def test_block_stage_by_stage(name, hidden):
    import paper_2505_16864_amd as J
    w = dict(ji.WORKLOADS[name], batch=2)
    d, heads = w["head_dim"], w["heads"]
    block, (w_qkv, b_qkv, w_out, b_out) = _block(w, hidden, 71)
    layer = block.layer
    x = randn(75, 2, block.tokens, hidden).to(torch.bfloat16)
    modulation = (0.3 * randn(76, 2, 6, hidden)).to(torch.bfloat16)                # scale and shift among a block's six vectors
    scale, shift = modulation[:, 1], modulation[:, 0]
    gpu = modulation.cuda()
    out = block.forward(x.cuda(), gpu[:, 1], gpu[:, 0])
    torch.cuda.synchronize()

    # norm and projection: 8-bit activations of a row are off by half a step of e4m3 (2^-4) of the value, no common sign
    xd = x.double()
    h = (xd - xd.mean(-1, keepdim=True)) / torch.sqrt(xd.var(-1, unbiased=False, keepdim=True) + 1e-6)
    y = (h * (1 + scale.double()[:, None]) + shift.double()[:, None]).reshape(-1, hidden)
    held = held_values(block.x, block.s_x, 1)
    # a scale rounded the other way at its border doubles the step
    assert bool(((held[:, :hidden] - y).abs() <= 2.0 ** -3 * y.abs() + 2.0 ** -9 * y.abs().amax(1, keepdim=True)).all())
    W = quantize(w_qkv.double(), 128)[0]
    assert torch.equal(held_values(block.w_qkv, block.s_qkv, 128), W)
    want = held @ W.t() + b_qkv.double()
    size = held.abs() @ W.abs().t() + b_qkv.double().abs()
    check(block.qkv.view(-1, 3 * heads * d), want, half_step(torch.bfloat16) * want.abs() * 1.01 + 8 * 2.0 ** -13 * size, "projection")

    # rotary positions and curve order
    lay = oracle_layout(w)
    dims = tuple(layer.rotary.dim)
    for t, got in ((0, layer.q_c), (1, layer.k_c)):
        src = block.qkv[:, :, t].cpu().double()
        turned = rotary(src, w["T"], w["H"], w["W"], dims, 256.0)
        top = src.abs().topk(2, dim=-1).values.sum(-1, keepdim=True)
        tol = half_step(torch.bfloat16) * turned.abs() + 4 * U32 * top
        to_curve = lambda a: torch.from_numpy(jo.permute(a.numpy(), lay))  # noqa: E731
        check(got, to_curve(turned), to_curve(tol), "turned")

    # attention over the tensors that the block made
    thw = [torch.empty_like(layer.out_thw) for _ in range(3)]
    for src, dst in zip((layer.q_c, layer.k_c, layer.v_c), thw):
        J.jenga_unpermute(layer.plan, src, dst)
    torch.cuda.synchronize()
    q, k, v = [ji.bits(t) for t in thw]
    attended, _, _ = jo.carve_layer(q, k, v, lay, w["p"])
    got = to_f64(layer.out_thw)
    check_output(np.swapaxes(got, 1, 2), np.swapaxes(attended, 1, 2), "attention")

    # output projection
    held = held_values(block.o, block.s_o, 1)
    assert torch.equal(held, quantize(torch.from_numpy(got).reshape(-1, heads * d), 1)[0])
    W = quantize(w_out.double(), 128)[0]
    want = held @ W.t() + b_out.double()
    size = held.abs() @ W.abs().t() + b_out.double().abs()
    check(out.view(-1, hidden), want, half_step(torch.bfloat16) * want.abs() * 1.01 + 8 * 2.0 ** -13 * size, "output")


# Captured once, replayed with new inputs, the program's own work between the replays; every replay against the eager result.
def test_block_in_a_graph():
    w = ji.WORKLOADS["tiny"]
    block, _ = _block(w, 256, 81)
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    inputs = [torch.randn((1, block.tokens, 256), generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(4)]
    want = [block.forward(x).clone() for x in inputs]
    x = inputs[0].clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block.forward(x)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.forward(x)
    for i in (1, 2, 3, 0, 2):
        x.copy_(inputs[i])
        graph.replay()
        got = block.out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, want[i]), i
        block.forward(inputs[(i + 1) % 4])                     # eager work of the same block between the replays
        torch.cuda.synchronize()
        assert torch.equal(block.out, want[(i + 1) % 4])


# Two blocks on two streams at once, each with its own buffers.
def test_two_blocks_on_two_streams():
    w = ji.WORKLOADS["small"]
    blocks = [_block(w, 512, 90 + i)[0] for i in range(2)]
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    x = [torch.randn((1, blocks[0].tokens, 512), generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(2)]
    want = [b.forward(t).clone() for b, t in zip(blocks, x)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for b in blocks:
            b.out.fill_(0)
        torch.cuda.synchronize()
        for b, t, s in zip(blocks, x, streams):
            with torch.cuda.stream(s):
                b.forward(t)
        torch.cuda.synchronize()
        assert all(torch.equal(b.out, t) for b, t in zip(blocks, want))


def test_block_refuses():
    from paper_2505_16864_amd.layer import CarveBlock
    w = ji.WORKLOADS["tiny"]
    inner = w["heads"] * w["head_dim"]
    good = (torch.zeros(3 * inner, 64), None, torch.zeros(64, inner), None)
    for bad in ((torch.zeros(2 * inner, 64),) + good[1:], good[:2] + (torch.zeros(64, inner + 1), None)):
        with pytest.raises(ValueError):
            CarveBlock(w, *bad, rotary=dict(dims=(16, 24, 24)))
    with pytest.raises(ValueError):
        CarveBlock(w, *good, rotary=None)
