"""Plain 64-bit forms of the norm without a mean, of 4-bit tensors and of dense attention, with what roundings may be off."""
import math

import torch

from operator_util import U32, half_step

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


# ---- the norm.  A sum of squares is off by n u of itself for n additions that follow each other: 24 values a lane, 6 steps across the wavefront and
# 16 wavefronts; rows too long for registers 128 values, 6 and 16 steps.  r = 1 / sqrt(..) has half of that and three roundings, y three more.
CHAIN = 150


def rms(total, w, w0, eps):
    """total float64 [..., cols] -> y, its slack before the last rounding, r."""
    r = 1 / torch.sqrt((total * total).mean(-1, keepdim=True) + eps)
    y = total * r * (w0 + w)
    return y, U32 * (CHAIN / 2 + 8) * y.abs(), r[..., 0]


def rms_grad(total, dy, w, w0, rstd, dtotal):
    """All float64 -> dx, its slack, dweight, its slack."""
    h, g = total * rstd[..., None], dy * (w0 + w)
    gh = g * h
    mean = gh.mean(-1, keepdim=True)
    dx = rstd[..., None] * (g - h * mean) + dtotal
    slack = U32 * (rstd[..., None] * (6 * g.abs() + h.abs() * ((CHAIN + 6) * gh.abs().mean(-1, keepdim=True) + 6 * mean.abs())) +
                   2 * dx.abs() + dtotal.abs())
    n = total.shape[-1]
    terms = (dy * h).reshape(-1, n)
    return dx, slack, terms.sum(0), U32 * (terms.shape[0] + 40) * terms.abs().sum(0)


# ---- 4-bit tensors

def e2m1_codes(v):
    """Codes of the nearest e2m1 values, ties to the even code."""
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    near = torch.round(a / step) * step
    code = torch.searchsorted(E2M1, near.contiguous())
    return (code + 8 * torch.signbit(v)).to(torch.uint8)


def quantize_mx(x):
    """x float64 [rows, cols] -> bytes [rows, C / 2], scales [rows, C / 32], as an exact quantisation gives them."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    full = torch.zeros((rows, padded), dtype=torch.float64)
    full[:, :cols] = x
    v = full.view(rows, padded // 32, 32)
    broken = ~torch.isfinite(v).all(2)
    largest = torch.where(broken, 0.0, v.abs().amax(2))
    m, e = torch.frexp(largest)                      # m in [1/2, 1); 6 = 3/4 * 2^3
    e = torch.where(m > 0.75, e - 2, e - 3)
    e = torch.where(largest == 0, 0, e).clamp(min=-127)
    unit = torch.ldexp(torch.ones_like(largest), e)[:, :, None]
    codes = torch.where(broken[:, :, None], 0, e2m1_codes(torch.where(broken[:, :, None], 0.0, v) / unit)).to(torch.uint8).view(rows, -1, 2)
    scale = torch.where(broken, 255, e + 127).to(torch.uint8)
    return codes[:, :, 0] | codes[:, :, 1] << 4, scale


def values_mx(q, scale):
    """What a 4-bit tensor stands for, float64 on the CPU."""
    q, scale = q.cpu(), scale.cpu()
    codes = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1, 32).long()
    v = E2M1[codes & 7] * torch.where(codes >= 8, -1.0, 1.0).double()
    unit = torch.ldexp(torch.ones(scale.shape, dtype=torch.float64), scale.int() - 127)
    unit = torch.where(scale == 255, math.nan, unit)
    return (v * unit[:, :, None]).view(q.shape[0], -1)


# ---- attention

def attention(q, k, v, q_lens, kv, causal, scale, dtype):
    """q [rows, heads, d], k, v [keys, kv_heads, d] of one type; kv: (start, length) of each sequence.  The result in float64 and how
    far a kernel's may be off: probabilities rounded to the type; logits of float32 sums of d products, and as arguments of the exponential
    three more roundings; sums over the keys; the result's rounding."""
    heads, group, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    out, tol, row = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), 0
    half = half_step(dtype)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0      # half a step among the smallest, of probabilities relative to one of 1 and of results
    for nq, (k0, nk) in zip(q_lens, kv):
        if nq and nk:
            for h in range(heads):
                qs, ks, vs = q[row:row + nq, h].double(), k[k0:k0 + nk, h // group].double(), v[k0:k0 + nk, h // group].double()
                sees = torch.ones(nq, nk, dtype=torch.bool)
                if causal:
                    sees = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq
                clean = torch.where(torch.isfinite(ks), ks, 0.0)
                s = (qs @ ks.t() if torch.isfinite(ks).all() else torch.stack([(qs[i][None] * ks).sum(1) for i in range(nq)])) * scale
                s = torch.where(sees, s, -math.inf)
                mags = torch.where(sees, (qs.abs() @ clean.abs().t()) * scale, 0.0)
                top = s.amax(1, keepdim=True)
                p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
                p = torch.where(sees, p, 0.0)
                total = p.sum(1, keepdim=True)
                some = total[:, 0] > 0
                p = p / torch.where(total > 0, total, 1.0)
                if torch.isfinite(vs).all():
                    o, a = p @ vs, p @ vs.abs()
                else:
                    o, a = [torch.stack([torch.where(sees[i][:, None], p[i][:, None] * t, 0.0).sum(0) for i in range(nq)]) for t in (vs, vs.abs())]
                delta = U32 * (d * mags.amax(1) + 6 * mags.amax(1) + 16)
                fine = torch.where(torch.isfinite(vs), vs.abs(), 0.0)
                err = a * (half + 2 * delta + 2 * (nk + 80) * U32)[:, None] * 1.01 + tiny * (sees.double() @ fine)
                out[row:row + nq, h] = torch.where(some[:, None], o, torch.where(sees.any(1)[:, None], o, 0.0))
                tol[row:row + nq, h] = err + half * (o.abs() + err) + tiny
        row += nq
    return out, tol
