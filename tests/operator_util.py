"""Plain 64-bit forms of the operators around the attention, and how far a rounding may be off."""
import math

import torch

U32 = 2.0 ** -24     # half a step of float32, relative
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def check(got, want, tol, what=""):
    """|got - want| <= tol value by value; NaN only where the other has it."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities in other places"
    err, tol = (got - want)[fine].abs(), tol.expand(want.shape)[fine]
    over = err > tol
    assert not over.any(), "%s: %d of %d values off, worst %.3g where %.3g is allowed" % (
        what, int(over.sum()), over.numel(), float(err[over].max()), float(tol[over][err[over].argmax()]))


# ---- 8-bit tensors

def e4m3(v):
    """Nearest e4m3 value of |v| <= 448, ties to even, in float64; NaN for what is not finite."""
    m, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    q = torch.round(v / step) * step
    return torch.where(torch.isfinite(v), q, torch.full_like(v, math.nan))


def quantize(x, block_rows):
    """x float64 [rows, cols] -> the values held [rows, C] times their scales, and the scale bytes [., S]."""
    rows, cols = x.shape
    blocks, padded_rows = -(-cols // 128), -(-rows // block_rows) * block_rows
    full = torch.zeros((padded_rows, blocks * 128), dtype=torch.float64)
    full[:rows, :cols] = x
    view = full.view(padded_rows // block_rows, block_rows, blocks, 128)
    finite = torch.where(torch.isfinite(view), view.abs(), torch.zeros_like(view))
    largest = finite.amax(dim=(1, 3))
    m, e = torch.frexp(largest)                      # m in [1/2, 1); 448 = 7/8 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(largest == 0, torch.zeros_like(e), e).clamp(min=-127)
    unit = torch.ldexp(torch.ones_like(largest), e)[:, None, :, None]
    held = (e4m3(view / unit) * unit).reshape(padded_rows, blocks * 128)[:rows]
    scale = torch.zeros((padded_rows // block_rows, -(-cols // 512) * 4), dtype=torch.uint8)
    scale[:, :blocks] = (e + 127).to(torch.uint8)
    return held, scale


def held_values(q, scale, block_rows):
    """What an 8-bit tensor stands for, float64 on the CPU."""
    q, scale = q.cpu(), scale.cpu()
    v = (q if q.dtype == torch.float8_e4m3fn else q.view(torch.float8_e4m3fn)).to(torch.float32).double()
    blocks = q.shape[1] // 128
    unit = torch.ldexp(torch.ones(scale.shape[0], blocks, dtype=torch.float64), scale[:, :blocks].int() - 127)
    return v * unit.repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(128, 1)


# ---- rotary

def rotary(x, T, H, W, dims, theta, origin=(0, 0, 0), step=(1, 1, 1), halves=False, inverse=False, cells=None):
    """x float64 [batch, tokens, heads, D]; cells int [batch, tokens, 3], -1: that axis is not turned; default: the grid's cells
    first, text behind."""
    batch, tokens = x.shape[:2]
    if cells is None:
        cells = torch.full((tokens, 3), -1, dtype=torch.int64)
        n = torch.arange(min(tokens, T * H * W))
        cells[:len(n)] = torch.stack([n // (H * W), n // W % H, n % W], 1)
        cells = cells.expand(batch, tokens, 3)
    out, at = x.clone(), 0
    for a, d in enumerate(dims):
        for i in range(d // 2):
            c0, c1 = (at + i, at + i + d // 2) if halves else (at + 2 * i, at + 2 * i + 1)
            cell = cells[..., a].clamp(max=(T, H, W)[a] - 1)
            angle = (origin[a] + step[a] * cell.double()) * theta ** (-2.0 * i / d)
            angle = torch.where(cell < 0, torch.zeros_like(angle), -angle if inverse else angle)[..., None]
            cos, sin = torch.cos(angle), torch.sin(angle)
            out[..., c0] = x[..., c0] * cos - x[..., c1] * sin
            out[..., c1] = x[..., c0] * sin + x[..., c1] * cos
        at += d
    return out
