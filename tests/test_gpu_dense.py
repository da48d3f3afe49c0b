"""jenga_dense_attn against float64, through the binding.  Tolerances: more_operator_util.attention."""
import pytest
import torch

from more_operator_util import attention
from operator_util import TYPES, check, randn

pytestmark = pytest.mark.gpu


def _starts(lengths):
    return torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), dtype=torch.int32, device="cuda:0")


def _room(q, k, sequences):
    import paper_2505_16864_amd as J
    size = J.jenga_dense_attn_workspace(q.shape[0], k.shape[0], sequences, q.shape[1], k.shape[1], q.shape[2])
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda:0")       # NaN, if any of it were read before it is written


def _run(q, k, v, q_lens, kv_lens, causal, **kw):
    import paper_2505_16864_amd as J
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda:0")
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    J.jenga_dense_attn(q, k, v, out, _starts(q_lens), _starts(kv_lens), causal=causal, workspace=_room(q, k, len(q_lens)), **kw)
    torch.cuda.synchronize()
    return out


def _inputs(rows, keys, heads, kv_heads, d, dtype, seed):
    t = TYPES[dtype]
    return (randn(seed, rows, heads, d).to(t), randn(seed + 1, keys, kv_heads, d).to(t),
            (randn(seed + 2, keys, kv_heads, d) + 0.5 * randn(seed + 3, kv_heads, d)).to(t))


def _kv(lengths):
    at, out = 0, []
    for n in lengths:
        out.append((at, n))
        at += n
    return out


CASES = [  # rows, keys of each sequence, heads, heads of keys
    ([1], [1], 1, 1), ([1], [0], 2, 1), ([1], [31], 5, 1), ([1], [33], 1, 1), ([1], [700], 8, 2), ([1] * 5, [1, 64, 129, 0, 1000], 10, 2),
    ([1] * 3, [4000, 10, 2500], 6, 6), ([2, 1, 3], [200, 130, 65], 4, 1), ([4], [300], 12, 3), ([7], [7], 1, 1), ([64], [64], 2, 2),
    ([128], [128], 1, 1), ([129], [129], 3, 1), ([33, 0, 200, 1, 90], [33, 12, 260, 70, 0], 6, 3), ([100], [40], 2, 2), ([40], [100], 2, 1),
    ([500, 60], [520, 700], 4, 4), ([300], [1200], 1, 1), ([65, 130], [65, 130], 10, 2), ([1000], [1000], 2, 1), ([250] * 4, [17, 300, 64, 65], 3, 3),
    ([17] * 9, [40] * 9, 16, 2), ([3000], [1], 2, 2), ([5, 0, 0], [5, 0, 9], 40, 8),
]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f16", 128), ("f16", 64)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_float64(case, causal, dtype, d):
    q_lens, kv_lens, heads, kv_heads = CASES[case]
    q, k, v = _inputs(sum(q_lens), sum(kv_lens), heads, kv_heads, d, dtype, case)
    want, tol = attention(q, k, v, q_lens, _kv(kv_lens), causal, d ** -0.5, q.dtype)
    check(_run(q, k, v, q_lens, kv_lens, causal), want, tol)


# Columns of one projection; rows off the 16-byte grid; heads in front of tokens; the result over q, or apart.
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [90, 300, 5]), ([150, 70], [150, 70])])
@pytest.mark.parametrize("d", [64, 128])
def test_strides(q_lens, kv_lens, d):
    import paper_2505_16864_amd as J
    heads, kv_heads, t = 6, 2, torch.bfloat16
    q, k, v = _inputs(sum(q_lens), sum(kv_lens), heads, kv_heads, d, "bf16", d)
    want, tol = attention(q, k, v, q_lens, _kv(kv_lens), True, 0.2, t)
    rows, keys = sum(q_lens), sum(kv_lens)
    starts, room = (_starts(q_lens), _starts(kv_lens)), _room(q, k, len(q_lens))

    def run(q, k, v, out, what):
        J.jenga_dense_attn(q, k, v, out, *starts, causal=True, scale=0.2, workspace=room)
        torch.cuda.synchronize()
        check(out, want, tol, what)

    wide = torch.full((max(rows, keys), heads + 2 * kv_heads, d), 5.0, dtype=t, device="cuda:0")
    wide[:rows, :heads], wide[:keys, heads:heads + kv_heads], wide[:keys, heads + kv_heads:] = q.cuda(), k.cuda(), v.cuda()
    parts = wide[:rows, :heads], wide[:keys, heads:heads + kv_heads], wide[:keys, heads + kv_heads:]
    run(*parts, torch.empty((rows, heads, d), dtype=t, device="cuda:0"), "columns")
    before = wide.clone()
    run(*parts, parts[0], "over q")
    assert torch.equal(wide[:, heads:], before[:, heads:]) and torch.equal(wide[rows:], before[rows:])
    odd = torch.full((max(rows, keys), (heads + 2 * kv_heads) * (d + 3) + 1), 5.0, dtype=t, device="cuda:0")
    odd = odd[:, 1:].unflatten(1, (heads + 2 * kv_heads, d + 3))
    odd[:rows, :heads, :d], odd[:keys, heads:heads + kv_heads, 1:d + 1], odd[:keys, heads + kv_heads:, 3:] = q.cuda(), k.cuda(), v.cuda()
    apart = torch.full((rows, heads, d + 1), 4.0, dtype=t, device="cuda:0")
    run(odd[:rows, :heads, :d], odd[:keys, heads:heads + kv_heads, 1:d + 1], odd[:keys, heads + kv_heads:, 3:], apart[:, :, 1:], "odd")
    assert bool((apart[:, :, 0] == 4).all())
    turned = [x.cuda().transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    run(*turned, torch.empty((heads, rows, d), dtype=t, device="cuda:0").transpose(0, 1), "heads in front")


# Keys in a cache with room behind each sequence, in another order than the rows, one of them of two sequences; the room holds NaN.
# Rows in front of the first sequence and behind the last are left as they were.
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [3, 70, 1, 200]])
def test_cache_with_room(q_lens):
    import paper_2505_16864_amd as J
    heads, kv_heads, d = 4, 2, 128
    lens, at = [300, 70, 300, 222], [800, 100, 800, 300]
    rows = sum(q_lens)
    q, k, v = _inputs(rows + 9, 1200, heads, kv_heads, d, "bf16", 3)
    used = torch.zeros(1200, dtype=torch.bool)
    for a, n in zip(at, lens):
        used[a:a + n] = True
    k[~used], v[~used] = float("nan"), float("nan")
    want, tol = attention(q[4:4 + rows], k, v, q_lens, list(zip(at, lens)), True, d ** -0.5, q.dtype)
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda:0")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    J.jenga_dense_attn(q.cuda(), k.cuda(), v.cuda(), out, _starts(q_lens) + 4, ints(at + [0]), kv_len=ints(lens), causal=True, workspace=_room(q, k, 4))
    torch.cuda.synchronize()
    check(out[4:4 + rows], want, tol)
    assert bool((out[:4] == 9).all()) and bool((out[4 + rows:] == 9).all())


# What a row does not see does not touch it: infinities and NaN in keys and values of later tokens and of other sequences.
@pytest.mark.parametrize("q_lens,kv_lens,heads,kv_heads", [([200, 100], [200, 100], 2, 1), ([6, 3], [40, 300], 2, 1), ([130], [400], 3, 3)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_what_is_not_seen(q_lens, kv_lens, heads, kv_heads, dtype, d):
    q, k, v = _inputs(sum(q_lens), sum(kv_lens), heads, kv_heads, d, dtype, 7)
    n = kv_lens[0]
    for i, bad in ((n - 1, float("nan")), (n - 3, float("inf")), (n - 2, -float("inf"))):
        v[i, 0, i % d] = bad
    k[n - 2, 0, 5] = float("nan")
    want, tol = attention(q, k, v, q_lens, _kv(kv_lens), True, d ** -0.5, q.dtype)
    got = _run(q, k, v, q_lens, kv_lens, True).cpu()
    seeing = q_lens[0] - 3                      # rows of the first sequence in front of all of these
    assert torch.isfinite(want[:seeing]).all() and torch.isfinite(want[q_lens[0]:]).all()
    for a, b in ((0, seeing), (q_lens[0], sum(q_lens))):
        check(got[a:b], want[a:b], tol[a:b])
    row = got[seeing, 0]                        # sees the infinity and nothing else of it
    assert bool(torch.isinf(row[(n - 3) % d])) and int(torch.isfinite(row).sum()) == d - 1
    assert bool(torch.isnan(got[q_lens[0] - 1, 0]).all())


# A key that makes NaN of a row does so however far its part's other logits lie below those of other parts.
@pytest.mark.parametrize("q_len", [1, 100])
def test_nan_among_small_logits(q_len):
    n = 4000
    q, k, v = _inputs(q_len, n, 1, 1, 64, "bf16", 21)
    q[:, 0, 0], k[:, 0, 0] = 4.0, 60.0
    k[:2000, 0, 0] = -60.0
    k[700, 0, 5] = float("nan")
    assert bool(torch.isnan(_run(q, k, v, [q_len], [n], False)).all())


# Logits that climb and fall along the keys by hundreds, so that the reference has to move, in either type; constant rows.
@pytest.mark.parametrize("q_len", [1, 150])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 128), ("f16", 64)])
def test_logits_far_apart(q_len, dtype, d):
    n = 1500
    q, k, v = _inputs(q_len, n, 2, 1, d, dtype, 11)
    ramp = torch.linspace(-60, 60, n, dtype=torch.float64)
    for form in (ramp, -ramp, 40 * torch.sin(ramp), torch.zeros(n, dtype=torch.float64)):
        k[:, 0, 0], q[:, :, 0] = form.to(k.dtype), 2.0
        want, tol = attention(q, k, v, [q_len], [(0, n)], False, 0.7, q.dtype)
        check(_run(q, k, v, [q_len], [n], False, scale=0.7), want, tol)


# The same call gives the same bits; a captured one follows its inputs, lengths among them, beside eager calls with a workspace of their own.
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [2000, 130, 900]), ([200, 333], [200, 900])])
def test_repeats_and_graph(q_lens, kv_lens):
    import paper_2505_16864_amd as J
    q, k, v = [x.cuda() for x in _inputs(sum(q_lens), sum(kv_lens), 10, 2, 128, "bf16", 5)]
    q_start, kv_start, room = _starts(q_lens), _starts(kv_lens), _room(q, k, len(q_lens))
    lens = torch.tensor(kv_lens, dtype=torch.int32, device="cuda:0")
    out = torch.empty_like(q)
    J.jenga_dense_attn(q, k, v, out, q_start, kv_start, kv_len=lens, causal=True, workspace=room)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        J.jenga_dense_attn(q, k, v, out, q_start, kv_start, kv_len=lens, causal=True, workspace=room)
    mine, other = _room(q, k, len(q_lens)), torch.empty_like(q)
    for i in range(4):
        q.copy_(randn(20 + i, *q.shape).to(q.dtype))
        lens.copy_(torch.tensor([max(1, n - 37 * i) for n in kv_lens], dtype=torch.int32))
        graph.replay()
        J.jenga_dense_attn(q, k, v, other, q_start, kv_start, kv_len=lens, causal=True, workspace=mine)
        torch.cuda.synchronize()
        assert torch.equal(out, other), i
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other), i


# Many sequences: more than the list of work keeps in LDS; empty ones between them.
def test_many_sequences():
    heads, d = 2, 64
    gen = torch.Generator().manual_seed(1)
    q_lens = torch.randint(0, 3, (5000,), generator=gen).tolist()
    kv_lens = torch.randint(0, 9, (5000,), generator=gen).tolist()
    q, k, v = _inputs(sum(q_lens), sum(kv_lens), heads, 1, d, "bf16", 1)
    want, tol = attention(q, k, v, q_lens, _kv(kv_lens), False, d ** -0.5, q.dtype)
    check(_run(q, k, v, q_lens, kv_lens, False), want, tol)


# Keys past 2^31 elements and 4 GiB of their tensors.
@pytest.mark.parametrize("q_len", [1, 200])
def test_far_keys(q_len):
    import paper_2505_16864_amd as J
    n, row, d = 300000, 7680, 128
    cache = torch.zeros((n, row), dtype=torch.bfloat16, device="cuda:0")
    q, k, v = _inputs(q_len, 2000, 1, 1, d, "bf16", 9)
    cache[-2000:, 7168:7296], cache[-2000:, 7296:7424] = k[:, 0].cuda(), v[:, 0].cuda()
    keys, values = cache[:, None, 7168:7296], cache[:, None, 7296:7424]
    out, ints = torch.empty(q.shape, dtype=q.dtype, device="cuda:0"), lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")
    J.jenga_dense_attn(q.cuda(), keys, values, out, ints([0, q_len]), ints([n - 2000, n]), causal=True, workspace=_room(q, keys, 1))
    torch.cuda.synchronize()
    want, tol = attention(q, k, v, [q_len], [(0, 2000)], True, d ** -0.5, q.dtype)
    check(out, want, tol)


# Starts and lengths that make no sense are cut to what is there.
@pytest.mark.parametrize("q_start,kv_start,kv_len", [
    ([-5, 30, 20, 1000], [0, 50, 40, 999999], None), ([0, 40, 0, 40], [-7, 90, 100, 60], None), ([3, 10, 40, 40], [90, 0, 500, 0], [1000, -3, 5])])
def test_malformed_starts(q_start, kv_start, kv_len):
    import paper_2505_16864_amd as J
    q, k, v = [x.cuda() for x in _inputs(40, 100, 4, 2, 64, "bf16", 2)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    out = torch.full_like(q, 9.0)
    J.jenga_dense_attn(q, k, v, out, ints(q_start), ints(kv_start), kv_len=None if kv_len is None else ints(kv_len), causal=True, workspace=_room(q, k, 3))
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
