"""Norms without a mean, 4-bit products and dense attention over packed sequences, as measurable cases.

Kinds of a case:

    rms        root-mean-square norm of each row (or of each head of a row) with a weight, after the addition of a residual or without.
    rms_train  the same forward and backward: the sum, the result, gradients of the sum and of the weight.
    matmul     rows of activations quantised to 4 bits (e2m1, a power-of-two scale for each 32 values) times a weight kept so.
    project    residual and norm straight to 8 or 4 bits, and the product with a weight of the same kind.
    attention  softmax attention over packed sequences of different lengths, causal or not, heads that share keys and values.

Where `own` is false the operators are computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rms(name, kind, rows, heads, cols, dtype, params, residual):
    case = {"kind": kind, "rows": rows, "heads": heads, "cols": cols, "dtype": dtype, "params": params, "residual": residual}
    return dict(case, name=name) if name else case


def _matmul(name, m, k, n, bias, out):
    case = {"kind": "matmul", "m": m, "k": k, "n": n, "bias": bias, "out": out}
    return dict(case, name=name) if name else case


def _project(name, m, k, n, bits):
    case = {"kind": "project", "m": m, "k": k, "n": n, "bits": bits}
    return dict(case, name=name) if name else case


def _attention(name, q, kv, heads, kv_heads, head_dim, dtype, causal):
    """q, kv: rows and keys of each sequence."""
    case = {"kind": "attention", "q": ",".join(map(str, q)), "kv": ",".join(map(str, kv)), "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "causal": causal}
    return dict(case, name=name) if name else case


def listed():
    prompts = [31, 512, 1024, 2000, 4096, 77, 8192, 333, 12000]
    cached = [1, 8192, 700, 4095, 2049, 33, 6000, 5121, 300, 1500, 4097, 64, 2777, 7001, 3333, 900]
    return [
        # one token: what a call costs
        _rms("rms_one_row", "rms", 1, 1, 5120, "bf16", "bf16", True),
        # Q and K of a 480p evaluation, each of 40 heads by itself, out of what one product for Q, K and V leaves
        _rms("rms_heads_480p", "rms", 33272, 40, 128, "bf16", "f32", False),
        # training in float32: two odd grids of tokens, columns off every power of two
        _rms("rms_train_odd", "rms_train", 12068, 1, 777, "f32", "f32", False),
        # fine-tuning on two clips, 12 heads x 128, with the residual stream and its gradient
        _rms("rms_train_clips", "rms_train", 63424, 1, 1536, "bf16", "bf16", True),
        # a weight read for a single row
        _matmul("mx4_one_row", 1, 1536, 9216, True, "bf16"),
        # sizes off every tile and block, the result in float32
        _matmul("mx4_odd", 777, 1000, 1111, False, "f32"),
        # Q, K and V of a 480p evaluation in one product
        _matmul("mx4_qkv_480p", 33272, 5120, 15360, True, "bf16"),
        # residual stream to Q, K and V, 31,200 tokens + 512 of text, 12 heads x 128, in 4 bits
        _project("project_mx4", 31712, 1536, 4608, 4),
        # one new token for each of 16 sequences over what is cached of them
        _attention("attn_tokens", [1] * len(cached), cached, 40, 8, 128, "bf16", True),
        # small odd sequences in half precision: one of no rows, rows that see no key, keys of earlier calls in front
        _attention("attn_odd", [1, 130, 0, 777, 64, 5], [500, 130, 9, 1201, 3, 0], 6, 3, 64, "f16", True),
        # two clips' tokens against their texts
        _attention("attn_cross", [31200, 31200], [512, 226], 12, 12, 128, "bf16", False),
        # whole prompts of very different lengths in one call
        _attention("attn_prompts", prompts, prompts, 40, 8, 128, "bf16", True),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["rms", "rms_train", "matmul", "matmul", "project", "attention", "attention", "attention"])
    if kind in ("rms", "rms_train"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        heads = rng.choice([1, 1, 1, 2, 5, 12, 40])
        cols = rng.choice([64, 72, 96, 128]) if heads > 1 else _log_uniform(rng, 64, 10000)
        if heads == 1 and rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        rows = _log_uniform(rng, 1, min(70000, (85000000 if dtype == "f32" else 170000000) // (heads * cols)))
        return _rms(None, kind, rows, heads, cols, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.6)
    if kind in ("matmul", "project"):
        while True:
            m, k, n = _log_uniform(rng, 1, 34000), _log_uniform(rng, 128, 14000), _log_uniform(rng, 64, 16000)
            if rng.random() < 0.6:
                k, n = max(128, k // 128 * 128), max(64, n // 64 * 64)
            if m * k * n <= 33272 * 5120 * 15360 and m * n <= 33272 * 15360:
                if kind == "project":
                    return _project(None, m, k, n, rng.choice([8, 4, 4]))
                return _matmul(None, m, k, n, rng.random() < 0.5, rng.choice(["bf16", "bf16", "f16", "f32"]))
    heads, kv_heads = rng.choice([(2, 2), (5, 1), (6, 3), (12, 12), (16, 2), (14, 2), (32, 8), (40, 40)])
    head_dim, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f16"])
    count = rng.choice([1, 2, 3, 5, 8, 17, 40])
    form = rng.choice(["prompts", "prompts", "tokens", "chunks", "cross"])
    while True:
        kv = [_log_uniform(rng, 1, 16000) for _ in range(count)]
        if form == "prompts":
            q = list(kv)
        elif form == "tokens":
            q = [1] * count
        elif form == "chunks":
            q = [rng.randint(0, n) for n in kv]
        else:
            q, kv = kv, [rng.randint(1, 700) for _ in range(count)]
        case = _attention(None, q, kv, heads, kv_heads, head_dim, dtype, form != "cross")
        if sum(q) > 0 and _pairs(case) * heads * head_dim * 4 <= 2.4e12 and max(sum(q), sum(kv)) * heads * head_dim <= 2e8:
            return case


# ---- inputs

def _hidden(gen, rows, cols, dtype):
    """Hidden states of a transformer: a spread and an offset of its own for each channel, a few channels far larger."""
    spread = torch.exp(0.4 * torch.randn(cols, generator=gen, device=DEVICE))
    spread = torch.where(torch.rand(cols, generator=gen, device=DEVICE) < 0.004, 20.0 * spread, spread)
    offset = 0.2 * torch.randn(cols, generator=gen, device=DEVICE)
    x = torch.randn((rows, cols), generator=gen, device=DEVICE)
    return x.mul_(spread).add_(offset).to(dtype)


def _lengths(case):
    return [int(n) for n in case["q"].split(",")], [int(n) for n in case["kv"].split(",")]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _pairs(case):
    """Rows and keys that see each other: the last row of a sequence sees all its keys, one before it a key less."""
    if not case["causal"]:
        return sum(a * b for a, b in zip(*_lengths(case)))
    total = 0
    for a, b in zip(*_lengths(case)):
        seeing = min(a, b)              # the rows that see a key at all see b - seeing + 1 to b of them
        total += seeing * (b - seeing) + seeing * (seeing + 1) // 2
    return total


def _width(k, block):
    return -(-k // block) * block


def _weight4(gen, n, k):
    """A weight [n, k] in 4 bits, its columns filled up with zeros, two values a byte, and its scale bytes."""
    w = torch.zeros((n, _width(k, 128)), device=DEVICE)
    w[:, :k] = torch.randn((n, k), generator=gen, device=DEVICE) / math.sqrt(k)
    v = w.view(n, -1, 32)
    e = _exponents(v.abs().amax(dim=2, keepdim=True), 6.0)
    a = v * _power(-e)
    size = torch.bucketize(a.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEVICE))   # a weight's ties may go down
    code = (size + 8 * (a < 0)).to(torch.uint8).view(n, -1, 2)
    return (code[:, :, 0] | code[:, :, 1] << 4).contiguous(), (e + 127).to(torch.uint8).view(n, -1).contiguous()


def _weight8(gen, n, k):
    """A weight [n, k] in e4m3 with a scale for each block of 128 x 128."""
    rows, padded = -(-n // 128), _width(k, 128)
    w = torch.zeros((rows * 128, padded), device=DEVICE)
    w[:n, :k] = torch.randn((n, k), generator=gen, device=DEVICE) / math.sqrt(k)
    e = _exponents(w.view(rows, 128, padded // 128, 128).abs().amax(dim=(1, 3)), 448.0)
    q = (w * _power(-e.repeat_interleave(128, 0).repeat_interleave(128, 1))).to(torch.float8_e4m3fn)[:n].contiguous()
    scale = torch.zeros((rows, _width(k, 512) // 128), dtype=torch.uint8, device=DEVICE)
    scale[:, :padded // 128] = (e + 127).to(torch.uint8)
    return q, scale


def _room(rows, k, bits):
    def empty(*shape):
        return torch.empty(shape, dtype=torch.uint8, device=DEVICE)
    if bits == 4:
        return empty(rows, _width(k, 128) // 2), empty(rows, _width(k, 128) // 32)
    return empty(rows, _width(k, 128)).view(torch.float8_e4m3fn), empty(rows, _width(k, 512) // 128)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, state = case["kind"], {"case": case}

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    if kind in ("rms", "rms_train"):
        rows, heads, cols, dtype = case["rows"], case["heads"], case["cols"], TYPES[case["dtype"]]
        if heads > 1:                                            # Q, K and V side by side in what one product leaves
            qkv = _hidden(gen, rows, 3 * heads * cols, dtype).view(rows, 3, heads, cols)
            xs, shape = [qkv[:, 0], qkv[:, 1]], (rows, heads, cols)
        else:
            xs, shape = [_hidden(gen, rows, cols, dtype)], (rows, cols)
        state["parts"] = []
        for x in xs:
            part = {"x": x, "weight": (1.0 + 0.3 * randn(cols)).to(TYPES[case["params"]]), "y": torch.empty(shape, dtype=dtype, device=DEVICE)}
            if case["residual"]:
                part.update(residual=randn(*shape).to(dtype), total=torch.empty(shape, dtype=dtype, device=DEVICE))
            if kind == "rms_train":
                part.update(dy=randn(*shape).to(dtype), dtotal=randn(*shape).to(dtype) if case["residual"] else None,
                            dx=torch.empty(shape, dtype=dtype, device=DEVICE), dweight=torch.empty(cols, device=DEVICE),
                            rstd=torch.empty(shape[:-1], device=DEVICE), room=None)
                if own:
                    import paper_2505_16864_amd as J
                    part["room"] = torch.empty(J.jenga_rms_norm_grad_workspace(rows * heads, cols), dtype=torch.uint8, device=DEVICE)
            state["parts"].append(part)
    elif kind in ("matmul", "project"):
        m, k, n = case["m"], case["k"], case["n"]
        bits = case.get("bits", 4)
        w, w_scale = (_weight4 if bits == 4 else _weight8)(gen, n, k)
        a, a_scale = _room(m, k, bits)
        state.update(x=_hidden(gen, m, k, torch.bfloat16), w=w, w_scale=w_scale, a=a, a_scale=a_scale,
                     bias=randn(n) if case.get("bias", True) else None,
                     out=torch.empty((m, n), dtype=TYPES[case.get("out", "bf16")], device=DEVICE))
        if kind == "project":
            state.update(residual=randn(m, k).to(torch.bfloat16), total=torch.empty((m, k), dtype=torch.bfloat16, device=DEVICE),
                         weight=(1.0 + 0.3 * randn(k)).to(torch.bfloat16))
    else:
        q_lens, kv_lens = _lengths(case)
        heads, kv_heads, d, dtype = case["heads"], case["kv_heads"], case["head_dim"], TYPES[case["dtype"]]
        if q_lens == kv_lens:                                    # columns of one projection
            qkv = randn(sum(q_lens), heads + 2 * kv_heads, d)
            qkv[:, heads + kv_heads:] += 0.5 * randn(kv_heads, d)
            q, k, v = qkv.to(dtype).split([heads, kv_heads, kv_heads], dim=1)
        else:
            q, k = randn(sum(q_lens), heads, d).to(dtype), randn(sum(kv_lens), kv_heads, d).to(dtype)
            v = (randn(sum(kv_lens), kv_heads, d) + 0.5 * randn(kv_heads, d)).to(dtype)
        starts = [torch.tensor(_starts(n), dtype=torch.int32, device=DEVICE) for n in (q_lens, kv_lens)]
        state.update(q=q, k=k, v=v, out=torch.empty(q.shape, dtype=dtype, device=DEVICE), q_start=starts[0], kv_start=starts[1], room=None)
        if own:
            import paper_2505_16864_amd as J
            size = J.jenga_dense_attn_workspace(sum(q_lens), sum(kv_lens), len(q_lens), heads, kv_heads, d)
            state["room"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)
    return state


# ---- the operators

EPS = 1e-6


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    import paper_2505_16864_amd as J
    case, kind = state["case"], state["case"]["kind"]
    if kind in ("rms", "rms_train"):
        out = []
        for p in state["parts"]:
            J.jenga_rms_norm(p["x"], p["y"], p["weight"], residual=p.get("residual"), total=p.get("total"), rstd=p.get("rstd"), eps=EPS)
            out += [p["total"], p["y"]] if case["residual"] else [p["y"]]
            if kind == "rms_train":
                total = p["total"] if case["residual"] else p["x"]
                J.jenga_rms_norm_grad(total, p["dy"], p["dx"], p["weight"], p["rstd"], dtotal=p["dtotal"], dweight=p["dweight"],
                                      workspace=p["room"])
                out += [p["dx"], p["dweight"]]
        return out
    if kind == "matmul":
        J.jenga_quantize_mx(state["x"], state["a"], state["a_scale"])
        J.jenga_matmul_mx(state["a"], state["a_scale"], state["w"], state["w_scale"], state["out"], state["bias"])
        return state["out"]
    if kind == "project":
        J.jenga_rms_norm(state["x"], state["a"], state["weight"], residual=state["residual"], total=state["total"],
                         y_scale=state["a_scale"], eps=EPS)
        product = J.jenga_matmul_mx if case["bits"] == 4 else J.jenga_matmul
        product(state["a"], state["a_scale"], state["w"], state["w_scale"], state["out"], state["bias"])
        return [state["total"], state["out"]]
    J.jenga_dense_attn(state["q"], state["k"], state["v"], state["out"], state["q_start"], state["kv_start"], causal=case["causal"],
                       workspace=state["room"])
    return state["out"]


def _plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind in ("rms", "rms_train"):
        out = []
        for p in state["parts"]:
            dtype, w = p["x"].dtype, p["weight"].float()
            total = _plain_total(p["x"], p.get("residual"))
            h, r = _plain_normed(total)
            out += [total, (h * w).to(dtype)] if case["residual"] else [(h * w).to(dtype)]
            if kind == "rms_train":
                dy = p["dy"].float()
                g = dy * w
                dx = r * (g - h * (g * h).mean(dim=-1, keepdim=True))
                if case["residual"]:
                    dx = dx + p["dtotal"].float()
                out += [dx.to(dtype), (dy * h).reshape(-1, case["cols"]).sum(dim=0)]
        return out
    if kind == "matmul":
        return _plain_product(state["x"].float(), state, 4)
    if kind == "project":
        total = _plain_total(state["x"], state["residual"])
        return [total, _plain_product(_plain_normed(total)[0] * state["weight"].float(), state, case["bits"])]
    return _plain_attention(state)


def _plain_total(x, residual):
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def _plain_normed(x):
    x = x.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    return x * r, r


def _exponents(largest, most):
    """The least e with largest <= most * 2^e, 0 where all values are zero (in 64 bits: the border has to be exact)."""
    mantissa, e = torch.frexp(largest.double() / most)
    return torch.where(largest == 0, 0, torch.where(mantissa == 0.5, e - 1, e)).clamp(-127, 127)


def _power(e):
    """2^e exactly, from the bits of the double (the device's own powers may be off by a last bit)."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _plain_e2m1(v):
    """The nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, ties to the one whose last bit is 0."""
    a = v.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.sign(v) * torch.round(a / step) * step


def _plain_product(x, state, bits):
    m, k = x.shape
    block, most = (32, 6.0) if bits == 4 else (128, 448.0)
    padded = torch.zeros((m, _width(k, 128) // block, block), device=DEVICE)
    padded.view(m, -1)[:, :k] = x
    e = _exponents(padded.abs().amax(dim=2, keepdim=True), most)
    a = padded * _power(-e)
    a = _plain_e2m1(a) if bits == 4 else a.to(torch.float8_e4m3fn).float()
    a = (a * _power(e)).view(m, -1)
    n = state["w"].shape[0]
    unit = _power(state["w_scale"][:, :a.shape[1] // block].int() - 127)
    if bits == 4:
        values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEVICE)
        code = torch.stack([state["w"] & 15, state["w"] >> 4], dim=2).view(n, -1).int()
        w = values[code & 7] * torch.where(code >= 8, -1.0, 1.0)
    else:
        w, unit = state["w"].float(), unit.repeat_interleave(128, 0)[:n]
    out = a @ (w.view(n, -1, block) * unit[:, :, None]).view(n, -1).t()
    return (out if state["bias"] is None else out + state["bias"]).to(state["out"].dtype)


def _plain_attention(state):
    case, out = state["case"], torch.zeros_like(state["out"])
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["head_dim"])
    q_lens, kv_lens = _lengths(case)
    for nq, nk, q0, k0 in zip(q_lens, kv_lens, _starts(q_lens), _starts(kv_lens)):
        if nq == 0 or nk == 0:
            continue
        k = state["k"][k0:k0 + nk].float().transpose(0, 1).contiguous()              # [kv_heads, keys, d]
        v = state["v"][k0:k0 + nk].float().transpose(0, 1).contiguous()
        most = max(1, (1 << 29) // (nk * group))                                     # rows at a time
        for r0 in range(0, nq, most):
            rows = min(most, nq - r0)
            q = state["q"][q0 + r0:q0 + r0 + rows].float()
            for h in range(case["kv_heads"]):
                s = q[:, h * group:(h + 1) * group].transpose(0, 1) @ k[h].t() * scale   # [group, rows, keys]
                if case["causal"]:
                    last = torch.arange(rows, device=DEVICE)[:, None] + (r0 + nk - nq)
                    s = s.masked_fill(torch.arange(nk, device=DEVICE)[None] > last, -math.inf)
                top = s.amax(dim=2, keepdim=True)
                p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
                total = p.sum(dim=2, keepdim=True)
                o = p @ v[h] / torch.where(total == 0, 1.0, total)
                out[q0 + r0:q0 + r0 + rows, h * group:(h + 1) * group] = o.transpose(0, 1).to(out.dtype)
    return out


def work(case):
    kind = case["kind"]
    if kind in ("rms", "rms_train"):
        size, parts = TYPES[case["dtype"]].itemsize, 2 if case["heads"] > 1 else 1
        values = case["rows"] * case["heads"] * case["cols"] * parts
        passes = 2 + (2 if case["residual"] else 0)                           # x and y; the residual and the sum
        if kind == "rms_train":
            passes += 2 + (1 if case["residual"] else 0)                      # dy and dx; the gradient that the sum gets from behind
        grads = 4 * case["cols"] * parts if kind == "rms_train" else 0
        return {"bytes": passes * values * size + parts * case["cols"] * TYPES[case["params"]].itemsize + grads,
                "flops": (5 if kind == "rms" else 14) * values}
    if kind in ("matmul", "project"):
        m, k, n, bits = case["m"], case["k"], case["n"], case.get("bits", 4)
        weight = n * k // 2 + n * k // 32 if bits == 4 else n * k
        bias = 4 * n if case.get("bias", True) else 0
        moved = (2 if kind == "matmul" else 6) * m * k + weight + bias + m * n * TYPES[case.get("out", "bf16")].itemsize
        return {"bytes": moved, "flops": 2 * m * n * k}
    q_lens, kv_lens = _lengths(case)
    d, size = case["head_dim"], TYPES[case["dtype"]].itemsize
    return {"bytes": size * d * (2 * sum(q_lens) * case["heads"] + 2 * sum(kv_lens) * case["kv_heads"]),
            "flops": 4 * _pairs(case) * case["heads"] * d}


# ---- the same from the definitions, in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rms", "rms_train"):
        return [o for p in state["parts"] for o in _exact_rms(p, case)]
    if kind == "matmul":
        return _exact_product(state["x"].double(), state, 4)
    if kind == "project":
        total, y = _exact_rms(state, {"residual": True, "kind": "rms"})
        return [total, _exact_product(y, state, case["bits"])]
    return _exact_attention(state)


def _exact_rms(p, case):
    """The sum is what a stream of this type holds of it; it is what is normed."""
    x, w = p["x"].double(), p["weight"].double()
    if case["residual"]:
        x = (x + p["residual"].double()).to(p["x"].dtype).double()
    n = x.shape[-1]
    length = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / n + EPS)
    y = x / length * w
    out = [x, y] if case["residual"] else [y]
    if case["kind"] == "rms_train":
        dy = p["dy"].double()
        along = (dy * w * x).sum(-1, keepdim=True) / (n * length ** 3)
        dx = dy * w / length - x * along
        out += [dx + p["dtotal"].double() if case["residual"] else dx, (dy * x / length).flatten(0, -2).sum(0)]
    return out


def _two_to(e):
    """2^e for whole e, from a list of Python's own powers."""
    powers = torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=DEVICE)
    return powers[(e + 300).long()]


def _rounded(v, bits):
    """Nearest value of 4 bits (two of exponent, one of mantissa) or 8 (four and three), ties to the even one."""
    least, places = (0, 1) if bits == 4 else (-6, 3)
    _, e = torch.frexp(v)
    step = _two_to((e - 1).clamp(min=least) - places)
    return torch.round(v / step) * step


def _exact_product(x, state, bits):
    block, top, most = (32, 0.75, 3) if bits == 4 else (128, 0.875, 9)       # 6 = 3/4 * 2^3, 448 = 7/8 * 2^9
    n, k = state["w"].shape[0], x.shape[1]
    a = torch.nn.functional.pad(x, (0, -k % 128)).view(x.shape[0], -1, block)
    m, e = torch.frexp(a.abs().amax(dim=2, keepdim=True))
    unit = _two_to(torch.where(m > 0, torch.where(m > top, e - most + 1, e - most), 0).clamp(min=-127))
    a = (_rounded(a / unit, bits) * unit).flatten(1)
    blocks = a.shape[1] // block
    unit = _two_to(state["w_scale"][:, :blocks].int() - 127)
    if bits == 4:
        sizes = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        table = torch.tensor([[_code(c & 15, sizes), _code(c >> 4, sizes)] for c in range(256)], dtype=torch.float64, device=DEVICE)
        w = table[state["w"].long()].view(n, blocks, block)
    else:
        w, unit = state["w"].double().view(n, blocks, block), unit[torch.arange(n, device=DEVICE) // 128]
    w = (w * unit[:, :, None]).flatten(1)
    out = torch.empty((x.shape[0], n), dtype=torch.float64, device=DEVICE)
    for c in range(0, n, 4096):
        out[:, c:c + 4096] = torch.mm(a, w[c:c + 4096].t())
    return out if state["bias"] is None else out.add_(state["bias"].double())


def _code(c, sizes):
    return -sizes[c - 8] if c >= 8 else sizes[c]


def _exact_attention(state):
    case = state["case"]
    group, out = case["heads"] // case["kv_heads"], torch.zeros(state["q"].shape, dtype=torch.float64, device=DEVICE)
    q_start, kv_start = [_starts(n) for n in _lengths(case)]
    for i in range(len(q_start) - 1):
        nq, nk = q_start[i + 1] - q_start[i], kv_start[i + 1] - kv_start[i]
        first = max(0, nq - nk) if case["causal"] else 0                     # rows before it see nothing
        if nk == 0 or first >= nq:
            continue
        k, v = [state[t][kv_start[i]:kv_start[i + 1]].double() for t in ("k", "v")]
        for h in range(case["heads"]):
            for r in range(first, nq, 2048):
                end = min(nq, r + 2048)
                seen = nk - nq + end if case["causal"] else nk               # by the last of these rows
                logits = torch.mm(state["q"][q_start[i] + r:q_start[i] + end, h].double(), k[:seen, h // group].t()) / case["head_dim"] ** 0.5
                if case["causal"]:
                    logits += torch.triu(torch.full_like(logits, -math.inf), diagonal=nk - nq + r + 1)
                out[q_start[i] + r:q_start[i] + end, h] = torch.mm(torch.softmax(logits, dim=1), v[:seen, h // group])
    return out
