"""The operators around a carved attention layer, as measurable cases.

Kinds of a case:

    norm        layer norm with a weight and a bias per group of rows: one group is the ordinary affine norm, a group per
                batch entry the modulation of a diffusion transformer (1 + scale, shift).
    norm_train  the same forward and backward: result, gradients of the input, the weight and the bias.
    matmul      rows of activations quantised to e4m3, a power-of-two scale for each 128 values, times a weight kept in e4m3
                with a scale for each block of 128 x 128.
    rotary      rotary positions over (time, height, width) on Q and K as a projection leaves them, text tokens as they are.
    project     hidden states to rotated Q, K and V: norm straight to e4m3, one product for all three, rotary in place.

Where `own` is false the operators are computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 128                # values that share a scale
E4M3_MAX = 448.0
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _norm(name, kind, rows, cols, groups, dtype, params):
    case = {"kind": kind, "rows": rows, "cols": cols, "groups": groups, "dtype": dtype, "params": params}
    return dict(case, name=name) if name else case


def _matmul(name, m, k, n, bias, out):
    case = {"kind": "matmul", "m": m, "k": k, "n": n, "bias": bias, "out": out}
    return dict(case, name=name) if name else case


def _rotary(name, T, H, W, n_text, batch, heads, head_dim, dims, theta, dtype, halves=False, inverse=False, step=1.0):
    case = {"kind": "rotary", "T": T, "H": H, "W": W, "n_text": n_text, "batch": batch, "heads": heads, "head_dim": head_dim,
            "dim_t": dims[0], "dim_h": dims[1], "dim_w": dims[2], "theta": theta, "dtype": dtype, "halves": halves,
            "inverse": inverse, "step": step}
    return dict(case, name=name) if name else case


def _project(name, T, H, W, n_text, heads, head_dim, dims, theta):
    case = {"kind": "project", "T": T, "H": H, "W": W, "n_text": n_text, "heads": heads, "head_dim": head_dim,
            "dim_t": dims[0], "dim_h": dims[1], "dim_w": dims[2], "theta": theta}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the tokens of the smallest grid in use, 2 heads x 64: what a call costs
        _norm("norm_tiny", "norm", 288, 128, 1, "bf16", "bf16"),
        # the modulated norm before the attention of a 480p evaluation: 32,760 tokens + 512 of text, 40 heads x 128
        _norm("norm_480p", "norm", 33272, 5120, 1, "bf16", "bf16"),
        # an ordinary affine norm in training in float32: two odd grids of tokens, columns off every power of two
        _norm("norm_train_odd", "norm_train", 12068, 777, 1, "f32", "f32"),
        # the modulated norm in fine-tuning: two clips, a weight and a bias for each, 12 heads x 128
        _norm("norm_train_clips", "norm_train", 63424, 1536, 2, "bf16", "bf16"),
        # the six modulation vectors of a block from one time-step embedding: a weight read for a single row
        _matmul("matmul_one_row", 1, 1536, 9216, True, "bf16"),
        # keys and values of the text tokens
        _matmul("matmul_text", 512, 5120, 10240, True, "bf16"),
        # sizes off every tile, the result in float32
        _matmul("matmul_odd", 777, 1000, 1111, False, "f32"),
        # Q, K and V of a 480p evaluation in one product
        _matmul("matmul_qkv_480p", 33272, 5120, 15360, True, "bf16"),
        # the smallest grid in use, head dim 64
        _rotary("rotary_tiny", 4, 8, 8, 32, 1, 2, 64, (16, 24, 24), 10000.0, "bf16"),
        # Q and K of a 720p evaluation, most of each head's channels for height and width
        _rotary("rotary_720p", 33, 45, 80, 256, 1, 24, 128, (16, 56, 56), 256.0, "bf16"),
        # the gradient for two odd grids in float32, halves of each axis' channels paired, positions of a coarser stage stretched
        _rotary("rotary_grad_odd", 7, 23, 37, 77, 2, 8, 64, (20, 22, 22), 10000.0, "f32", True, True, 1.25),
        # hidden states to rotated Q, K and V, 31,200 tokens + 512 of text, 12 heads x 128; axes that share 16-byte pieces
        _project("project_480p_small", 20, 30, 52, 512, 12, 128, (44, 42, 42), 10000.0),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _grid(rng, most):
    """A grid of up to `most` tokens: 1 to 33 frames, any aspect ratio between 1 and 2."""
    tokens = _log_uniform(rng, 24, most)
    T = max(1, min(33, round(tokens ** (1.0 / 3.0) * rng.uniform(0.5, 1.2))))
    H = max(1, round(math.sqrt(tokens / T / rng.uniform(1.0, 2.0))))
    return T, H, max(1, int(tokens / T / H))


def _axes(rng, head_dim):
    """Even channel counts of the three axes; now and then some channels keep their place."""
    t = 2 * rng.randint(0, head_dim // 8)
    h = 2 * rng.randint(1, (head_dim - t) // 4)
    w = head_dim - t - h if rng.random() < 0.7 else 2 * rng.randint(1, (head_dim - t - h) // 2)
    return t, h, w


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "matmul", "matmul", "matmul", "rotary", "rotary", "project"])
    if kind in ("norm", "norm_train"):
        cols = _log_uniform(rng, 64, 8192)
        rows = _log_uniform(rng, 1, min(120000, 170000000 // cols))
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        groups = min(rows, rng.choice([1, 1, 2, 5]))
        return _norm(None, kind, rows // groups * groups, cols, groups, dtype, rng.choice([dtype, "f32"]))
    if kind == "matmul":
        while True:
            m, k, n = _log_uniform(rng, 1, 34000), _log_uniform(rng, 128, 14000), _log_uniform(rng, 64, 16000)
            if rng.random() < 0.6:
                k, n = max(128, k // 128 * 128), max(64, n // 64 * 64)
            if m * k * n <= 33272 * 5120 * 15360 and m * n <= 33272 * 15360:
                return _matmul(None, m, k, n, rng.random() < 0.5, rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "rotary":
        head_dim = rng.choice([64, 128, 128, 96, 72])
        heads = rng.choice([2, 3, 8, 12, 24, 40])
        batch = rng.choice([1, 1, 2, 3])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        grid = _grid(rng, min(118800, 680000000 // (batch * heads * head_dim * TYPES[dtype].itemsize)))
        return _rotary(None, *grid, rng.choice([0, 1, 32, 77, 256]), batch, heads, head_dim, _axes(rng, head_dim),
                       rng.choice([256.0, 10000.0]), dtype, rng.random() < 0.4, rng.random() < 0.4, rng.choice([1.0, 0.75, 1.25]))
    heads, head_dim = rng.choice([2, 3, 8, 12, 40]), rng.choice([64, 128])
    grid = _grid(rng, 30000)
    return _project(None, *grid, rng.choice([0, 5, 77, 256]), heads, head_dim, _axes(rng, head_dim), rng.choice([256.0, 10000.0]))


# ---- inputs

def _hidden(gen, rows, cols, dtype):
    """Hidden states of a transformer: a spread and an offset of its own for each channel, a few channels far larger."""
    spread = torch.exp(0.4 * torch.randn(cols, generator=gen, device=DEVICE))
    spread = torch.where(torch.rand(cols, generator=gen, device=DEVICE) < 0.004, 20.0 * spread, spread)
    offset = 0.2 * torch.randn(cols, generator=gen, device=DEVICE)
    x = torch.randn((rows, cols), generator=gen, device=DEVICE)
    return x.mul_(spread).add_(offset).to(dtype)


def _tokens(case):
    return case["T"] * case["H"] * case["W"] + case["n_text"]


def _quantised_weight(gen, n, k):
    """A weight [n, k] in e4m3, its columns filled up with zeros to whole blocks, and its scale bytes: what a program keeps."""
    padded = -(-k // BLOCK) * BLOCK
    rows = -(-n // BLOCK)
    w = torch.zeros((rows * BLOCK, padded), device=DEVICE)
    w[:n, :k] = torch.randn((n, k), generator=gen, device=DEVICE) / math.sqrt(k)
    e = _exponents(w.view(rows, BLOCK, padded // BLOCK, BLOCK).abs().amax(dim=(1, 3)))
    spread = e.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)
    q = (w * _power(-spread)).to(torch.float8_e4m3fn)[:n].contiguous()
    scale = torch.zeros((rows, _scale_columns(k)), dtype=torch.uint8, device=DEVICE)
    scale[:, :padded // BLOCK] = (e + 127).to(torch.uint8)
    return q, scale


def _scale_columns(k):
    return -(-k // (4 * BLOCK)) * 4     # bytes of a row of scales: whole groups of four


def _quantised_room(rows, k):
    padded = -(-k // BLOCK) * BLOCK
    return (torch.empty((rows, padded), dtype=torch.float8_e4m3fn, device=DEVICE),
            torch.empty((rows, _scale_columns(k)), dtype=torch.uint8, device=DEVICE))


def _rotary_table(case):
    """(cos, sin) of every pair of every cell of each axis, one axis behind the other: [pairs, 2] in float32."""
    parts = []
    for cells, d in ((case["T"], case["dim_t"]), (case["H"], case["dim_h"]), (case["W"], case["dim_w"])):
        freq = float(case["theta"]) ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / max(d, 1))
        angle = (case.get("step", 1.0) * torch.arange(cells, dtype=torch.float64)[:, None] * freq).reshape(-1)
        parts.append(torch.stack([torch.cos(angle), torch.sin(angle)], dim=1))
    return torch.cat(parts).to(torch.float32).to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, state = case["kind"], {"case": case}

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    if kind in ("norm", "norm_train"):
        rows, cols, dtype, params = case["rows"], case["cols"], TYPES[case["dtype"]], TYPES[case["params"]]
        x = _hidden(gen, rows, cols, dtype)
        state.update(x=x, weight=(0.3 * randn(case["groups"], cols)).to(params), bias=(0.3 * randn(case["groups"], cols)).to(params),
                     y=torch.empty_like(x))
        if kind == "norm_train":
            grads = [torch.empty((case["groups"], cols), device=DEVICE) for _ in range(2)]
            room = torch.empty((1024 + case["groups"]) * cols * 8, dtype=torch.uint8, device=DEVICE)
            state.update(dy=randn(rows, cols).to(dtype), dx=torch.empty_like(x), dweight=grads[0], dbias=grads[1], room=room,
                         mean=torch.empty(rows, device=DEVICE), rstd=torch.empty(rows, device=DEVICE))
    elif kind == "matmul":
        m, k, n = case["m"], case["k"], case["n"]
        w, w_scale = _quantised_weight(gen, n, k)
        a, a_scale = _quantised_room(m, k)
        state.update(x=_hidden(gen, m, k, torch.bfloat16), w=w, w_scale=w_scale, bias=randn(n) if case["bias"] else None, a=a,
                     a_scale=a_scale, out=torch.empty((m, n), dtype=TYPES[case["out"]], device=DEVICE))
    elif kind == "rotary":
        # Q and K side by side in what one product leaves: [batch, tokens, 3, heads, head_dim]
        shape = (case["batch"], _tokens(case), 3, case["heads"], case["head_dim"])
        dtype = TYPES[case["dtype"]]
        qkv = torch.empty(shape, dtype=dtype, device=DEVICE)
        for b in range(shape[0]):
            qkv[b] = randn(*shape[1:]).to(dtype)
        out = [torch.empty(shape[:2] + shape[3:], dtype=dtype, device=DEVICE) for _ in range(2)]
        state.update(q=qkv[:, :, 0], k=qkv[:, :, 1], q_out=out[0], k_out=out[1], table=_rotary_table(case))
    else:
        rows, cols = _tokens(case), case["heads"] * case["head_dim"]
        w, w_scale = _quantised_weight(gen, 3 * cols, cols)
        a, a_scale = _quantised_room(rows, cols)
        state.update(x=_hidden(gen, rows, cols, torch.bfloat16), weight=(0.3 * randn(1, cols)).to(torch.bfloat16),
                     bias=(0.3 * randn(1, cols)).to(torch.bfloat16), w=w, w_scale=w_scale, w_bias=0.1 * randn(3 * cols), a=a,
                     a_scale=a_scale, qkv=torch.empty((rows, 3 * cols), dtype=torch.bfloat16, device=DEVICE), table=_rotary_table(case))
    return state


# ---- the operators

EPS = 1e-6


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    import paper_2505_16864_amd as J
    case = state["case"]
    kind, stream = case["kind"], torch.cuda.current_stream().cuda_stream
    if kind in ("norm", "norm_train"):
        x, group_rows = state["x"], case["rows"] // case["groups"]
        if kind == "norm":
            J.jenga_layer_norm(x, state["y"], state["weight"], state["bias"], group_rows=group_rows, weight_offset=1.0, eps=EPS,
                               stream=stream)
            return state["y"]
        J.jenga_layer_norm(x, state["y"], state["weight"], state["bias"], mean=state["mean"], rstd=state["rstd"],
                           group_rows=group_rows, weight_offset=1.0, eps=EPS, stream=stream)
        J.jenga_layer_norm_grad(x, state["dy"], state["dx"], state["weight"], state["mean"], state["rstd"], state["dweight"],
                                state["dbias"], state["room"], group_rows=group_rows, weight_offset=1.0, stream=stream)
        return [state["y"], state["dx"], state["dweight"], state["dbias"]]
    if kind == "matmul":
        J.jenga_quantize(state["x"], state["a"], state["a_scale"], stream=stream)
        J.jenga_matmul(state["a"], state["a_scale"], state["w"], state["w_scale"], state["out"], state["bias"], stream=stream)
        return state["out"]
    flags = (J.JENGA_ROTARY_HALVES if case.get("halves") else 0) | (J.JENGA_ROTARY_INVERSE if case.get("inverse") else 0)
    config = J.make_rotary(case["T"], case["H"], case["W"], case["head_dim"], (case["dim_t"], case["dim_h"], case["dim_w"]),
                           case["theta"], step=(case.get("step", 1.0),) * 3, flags=flags)
    if kind == "rotary":
        J.jenga_rotary(config, state["table"], state["q"], state["q_out"], state["k"], state["k_out"], stream=stream)
        return [state["q_out"], state["k_out"]]
    J.jenga_layer_norm(state["x"], state["a"], state["weight"], state["bias"], y_scale=state["a_scale"], weight_offset=1.0, eps=EPS,
                       stream=stream)
    J.jenga_matmul(state["a"], state["a_scale"], state["w"], state["w_scale"], state["qkv"], state["w_bias"], stream=stream)
    q, k, v = state["qkv"].view(1, -1, 3, case["heads"], case["head_dim"]).unbind(2)
    J.jenga_rotary(config, state["table"], q, q, k, k, stream=stream)
    return state["qkv"]


def _plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        h, r = _plain_normed(state["x"])
        w, b = [_per_row(state[p], case).float() for p in ("weight", "bias")]
        y = (h * (1.0 + w) + b).to(state["x"].dtype)
        if kind == "norm":
            return y
        dy = state["dy"].float()
        g = dy * (1.0 + w)
        dx = r * (g - g.mean(dim=1, keepdim=True) - h * (g * h).mean(dim=1, keepdim=True))
        return [y, dx.to(state["x"].dtype), _group_sums(dy * h, case), _group_sums(dy, case)]
    if kind == "matmul":
        return _plain_matmul(state["x"].float(), state["w"], state["w_scale"], state["bias"], state["out"].dtype)
    if kind == "rotary":
        return [_plain_rotary(state[t], state["table"], case).to(state[t].dtype) for t in ("q", "k")]
    h, _ = _plain_normed(state["x"])
    a = h * (1.0 + state["weight"].float()) + state["bias"].float()
    qkv = _plain_matmul(a, state["w"], state["w_scale"], state["w_bias"], torch.bfloat16)
    qkv = qkv.view(1, -1, 3, case["heads"], case["head_dim"])
    turned = [_plain_rotary(qkv[:, :, t], state["table"], case).to(torch.bfloat16) for t in (0, 1)]
    return torch.stack(turned + [qkv[:, :, 2]], dim=2).reshape(state["qkv"].shape)


def _plain_normed(x):
    x = x.float()
    d = x - x.mean(dim=1, keepdim=True)
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    return d * r, r


def _per_row(p, case):
    return p if case["groups"] == 1 else p.repeat_interleave(case["rows"] // case["groups"], 0)


def _group_sums(x, case):
    return x.view(case["groups"], -1, x.shape[1]).sum(dim=1)


def _exponents(largest):
    """The least e with largest <= 448 * 2^e, 0 where all values are zero (in 64 bits: the border has to be exact)."""
    mantissa, e = torch.frexp(largest.double() / E4M3_MAX)
    return torch.where(largest == 0, 0, torch.where(mantissa == 0.5, e - 1, e)).clamp(-127, 127)


def _power(e):
    """2^e exactly, from the bits of the double (the device's own powers may be off by a last bit)."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _plain_matmul(x, w, w_scale, bias, dtype):
    m, k = x.shape
    blocks = w.shape[1] // BLOCK
    padded = torch.zeros((m, blocks, BLOCK), device=DEVICE)
    padded.view(m, -1)[:, :k] = x
    e = _exponents(padded.abs().amax(dim=2, keepdim=True))
    a = ((padded * _power(-e)).to(torch.float8_e4m3fn).float() * _power(e)).view(m, -1)
    scale = _power(w_scale[:, :blocks].int() - 127).repeat_interleave(BLOCK, 0)[:w.shape[0]]
    b = (w.float().view(-1, blocks, BLOCK) * scale[:, :, None]).view(w.shape)
    out = a @ b.t()
    return (out if bias is None else out + bias).to(dtype)


def _pair_places(case):
    """For each pair of channels: its two channels, its axis and its place in that axis."""
    d = torch.tensor([case["dim_t"], case["dim_h"], case["dim_w"]], device=DEVICE)
    axis = torch.arange(3, device=DEVICE).repeat_interleave(d // 2)
    start = (torch.cumsum(d, 0) - d)[axis]                                     # the axis' first channel
    place = torch.arange(len(axis), device=DEVICE) - start // 2
    if case.get("halves"):
        return start + place, start + place + (d // 2)[axis], axis, place
    return start + 2 * place, start + 2 * place + 1, axis, place


def _plain_rotary(x, table, case):
    T, H, W = case["T"], case["H"], case["W"]
    first, second, axis, place = _pair_places(case)
    n = torch.arange(T * H * W, device=DEVICE)
    cells = torch.stack([n // (H * W), n // W % H, n % W], dim=1)
    pairs = torch.tensor([case["dim_t"] // 2, case["dim_h"] // 2, case["dim_w"] // 2], device=DEVICE)
    rows = torch.tensor([T, H, W], device=DEVICE) * pairs
    at = (torch.cumsum(rows, 0) - rows)[axis] + cells[:, axis] * pairs[axis] + place
    cos, sin = table[at][:, None, :, 0], table[at][:, None, :, 1]
    if case.get("inverse"):
        sin = -sin
    out = x.float().clone()
    u, v = out[:, :T * H * W, :, first], out[:, :T * H * W, :, second]
    out[:, :T * H * W, :, first] = u * cos - v * sin
    out[:, :T * H * W, :, second] = u * sin + v * cos
    return out


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        size = TYPES[case["dtype"]].itemsize
        values, params = case["rows"] * case["cols"], case["groups"] * case["cols"]
        passes = 2 if kind == "norm" else 4              # x and y; dy and dx too
        grads = 0 if kind == "norm" else 8 * params
        return {"bytes": passes * values * size + 2 * params * TYPES[case["params"]].itemsize + grads,
                "flops": (8 if kind == "norm" else 20) * values}
    if kind == "matmul":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": 2 * m * k + n * k + m * n * TYPES[case["out"]].itemsize + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    values = _tokens(case) * case["heads"] * case["head_dim"]
    if kind == "rotary":
        return {"bytes": 4 * case["batch"] * values * TYPES[case["dtype"]].itemsize, "flops": 6 * case["batch"] * values}
    cols = case["heads"] * case["head_dim"]
    return {"bytes": 2 * values + 3 * cols * cols + 6 * values, "flops": 6 * values * cols + 14 * values}


# ---- the same from the definitions, in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "matmul":
        return _exact_product(state["x"].double(), state)
    if kind == "rotary":
        return [_exact_turned(state[t].double(), case) for t in ("q", "k")]
    x = state["x"].double()
    groups = case.get("groups", 1)
    size = x.shape[0] // groups
    parts = [_exact_norm(x[g * size:(g + 1) * size], state["weight"][g].double(), state["bias"][g].double(),
                         state["dy"][g * size:(g + 1) * size].double() if kind == "norm_train" else None) for g in range(groups)]
    y = torch.cat([p[0] for p in parts])
    if kind == "norm":
        return y
    if kind == "norm_train":
        return [y, torch.cat([p[1] for p in parts]), torch.stack([p[2] for p in parts]), torch.stack([p[3] for p in parts])]
    out = _exact_product(y, {"w": state["w"], "w_scale": state["w_scale"], "bias": state["w_bias"]})
    out = out.view(1, -1, 3, case["heads"], case["head_dim"])
    for t in (0, 1):
        out[:, :, t] = _exact_turned(out[:, :, t], case)
    return out.view(state["qkv"].shape)


def _exact_norm(x, w, b, dy):
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    sd = torch.sqrt(var + EPS)
    h = (x - mean) / sd
    y = torch.addcmul(b, h, w + 1.0)
    if dy is None:
        return [y]
    g = dy * (w + 1.0)
    n = x.shape[1]
    dx = (g - (g.sum(1, True) + h * torch.einsum("rc,rc->r", g, h)[:, None]) / n) / sd
    return [y, dx, torch.einsum("rc,rc->c", dy, h), dy.sum(0)]


def _two_to(e):
    """2^e for whole e, from a list of Python's own powers."""
    powers = torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=DEVICE)
    return powers[(e + 300).long()]


def _e4m3(v):
    """Nearest value of four exponent and three mantissa bits, ties to the even one."""
    _, e = torch.frexp(v)
    step = _two_to((e - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _exact_product(x, state):
    w = state["w"].double()
    n, k = w.shape
    out = torch.zeros((x.shape[0], n), dtype=torch.float64, device=DEVICE)
    for at in range(0, k, BLOCK):
        part = x[:, at:at + BLOCK]
        largest = part.abs().amax(dim=1, keepdim=True)
        m, e = torch.frexp(largest)                          # largest = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
        unit = _two_to(torch.where(largest > 0, torch.where(m > 0.875, e - 8, e - 9), 0).clamp(min=-127))
        block = w[:, at:at + part.shape[1]] * _two_to(state["w_scale"][:, at // BLOCK].int() - 127).repeat_interleave(BLOCK)[:n, None]
        out.addmm_(_e4m3(part / unit) * unit, block.t())
    return out if state["bias"] is None else out.add_(state["bias"].double())


def _exact_turned(x, case):
    """Each pair of channels as a complex number, times e^(i angle)."""
    out, start = x.clone(), 0
    grid = x[:, :case["T"] * case["H"] * case["W"]]
    for d, cells, inner in ((case["dim_t"], case["T"], case["H"] * case["W"]), (case["dim_h"], case["H"], case["W"]), (case["dim_w"], case["W"], 1)):
        if d:
            part = grid[..., start:start + d]
            pairs = torch.stack([part[..., :d // 2], part[..., d // 2:]], -1) if case.get("halves") else part.reshape(*part.shape[:-1], d // 2, 2)
            cell = torch.arange(grid.shape[1], device=DEVICE) // inner % cells
            rate = torch.exp(-math.log(case["theta"]) * 2.0 / d * torch.arange(d // 2, device=DEVICE, dtype=torch.float64))
            angle = (cell.double() * case.get("step", 1.0))[:, None, None] * rate
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), -angle if case.get("inverse") else angle))
            out[:, :grid.shape[1], :, start:start + d] = torch.cat([turned[..., 0], turned[..., 1]], -1) if case.get("halves") else turned.reshape(part.shape)
        start += d
    return out
