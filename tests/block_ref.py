"""The transformer-block operators from their definitions, in 64 bits, with bounds on what the kernels may be off: every rounding
on the way counted at half a step of its type (relative 2^-24 for fp32, 2^-8 for bf16)."""
import math

import torch

F32, BF16 = 2.0 ** -24, 2.0 ** -8


def half_step(dtype):
    return BF16 if dtype == torch.bfloat16 else F32


def attention(q, k, v, lens, scale):
    """(o, bound) in float64.  A score is a sum of D fp32 products and two more roundings: off by (D + 4) 2^-24 scale sum |q_i k_i|
    at most, and its exponential by 2^-18 more.  Sums over n keys add n 2^-24.  All of that hits numerator and denominator.  bf16
    rounds each probability (numerator only), and the result is rounded once."""
    b, t, h, d = q.shape
    n, hkv = k.shape[1], k.shape[2]
    qd, kd, vd = (x.double() for x in (q, k, v))
    o, bound = torch.zeros_like(qd), torch.zeros_like(qd)
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        if m == 0:
            continue
        kk, vv = kd[i, :m].repeat_interleave(h // hkv, 1), vd[i, :m].repeat_interleave(h // hkv, 1)
        s = scale * torch.einsum("thd,uhd->htu", qd[i], kk)
        p = torch.softmax(s, 2)
        o[i] = torch.einsum("htu,uhd->thd", p, vv)
        spread = torch.einsum("htu,uhd->thd", p, vv.abs())
        off = (d + 4) * F32 * scale * torch.einsum("thd,uhd->htu", qd[i].abs(), kk.abs()).amax() + 2.0 ** -18 + (m + 16) * F32
        bound[i] = (2 * off + (BF16 if q.dtype == torch.bfloat16 else 0.0)) * spread
    return o, bound + half_step(q.dtype) * (o.abs() + bound)


def rotary(x, freqs, positions, pairs, layout, amplitude=1.0):
    """(y, bound) in float64.  sin and cos are off by 2^-21 at most: the angle in turns is rounded to fp32 (2^-26 of a turn, times
    2 pi), then the function's own two units of 2^-24, and the amplitude's product."""
    r = 2 * freqs.numel()
    xd = x.double()
    at = positions.double().repeat_interleave(torch.tensor(pairs, device=x.device), dim=2, output_size=r // 2)
    turns = at * freqs.to(x.device)
    angle = (2 * math.pi * (turns - turns.round())).unsqueeze(2)
    cos, sin = amplitude * angle.cos(), amplitude * angle.sin()
    y, off = xd.clone(), torch.zeros_like(xd)
    one, two = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    u, w = xd[..., one], xd[..., two]
    y[..., one], y[..., two] = u * cos - w * sin, u * sin + w * cos
    off[..., one] = off[..., two] = (u.abs() + w.abs()) * max(abs(amplitude), 1e-30) * (2.0 ** -21 + 2 * F32)
    turned = torch.zeros(x.shape[3], dtype=torch.bool, device=x.device)
    turned[:r] = True
    return y, torch.where(turned, off + half_step(x.dtype) * (y.abs() + off), 0.0)


SUM = 160 * F32          # a sum over a token: at most 128 additions in a row (per thread, warp and block) and the roundings around them


def _unit(z, dz, kind, eps):
    """norm(z), and what it may be off where z is off by dz."""
    mean = z.mean(2, keepdim=True) if kind == "layer" else 0.0
    rstd = torch.rsqrt((z - mean).square().mean(2, keepdim=True) + eps)
    u = (z - mean) * rstd
    dm = (SUM * z.abs().mean(2, keepdim=True) if kind == "layer" else 0.0) + dz.amax(2, keepdim=True)
    return u, rstd * dm * (2 + u.abs()) + 4 * SUM * u.abs()


def gate_norm(x, h=None, gate=None, scale=None, shift=None, kind="layer", eps=1e-6, weight=None, bias=None, post_norm=False, post_weight=None,
              residual_scale=1.0, mod_tokens=None, x_dtype=None, y_dtype=None):
    """(r, bound, y, bound) in float64."""
    t = x.shape[1]
    rows = torch.arange(t, device=x.device) // (mod_tokens or max(t, 1))
    at = lambda m, other: torch.full((), other, dtype=torch.float64, device=x.device) if m is None else m.double()[:, rows]
    one = lambda w: torch.ones((), dtype=torch.float64, device=x.device) if w is None else w.double()
    r, dr = x.double(), torch.zeros_like(x, dtype=torch.float64)
    if h is not None:
        u, du = h.double(), torch.zeros_like(dr)
        if post_norm:
            u, du = _unit(u, du, kind, eps)
        f = residual_scale * at(gate, 1.0) * one(post_weight)
        dr = f.abs() * du + 4 * F32 * ((f * u).abs() + r.abs())
        r = r + f * u
    z, dz = _unit(r, dr, kind, eps)
    g = 1 + at(scale, 0.0)
    base = z * one(weight) + (0.0 if bias is None else bias.double())
    y = base * g + at(shift, 0.0)
    dy = (one(weight) * g).abs() * dz + 8 * F32 * (((z * one(weight)).abs() + (base.abs())) * (1 + g.abs()) + y.abs() + at(shift, 0.0).abs())
    return r, dr + half_step(x_dtype or x.dtype) * (r.abs() + dr), y, dy + half_step(y_dtype or (x if h is None else h).dtype) * (y.abs() + dy)


def check(got, want, bound):
    g = got.double()
    assert torch.isfinite(g).all()
    off = (g - want).abs() - bound
    assert (off <= 1e-30).all(), f"{int((off > 1e-30).sum())} of {off.numel()} values beyond their bound, the worst at {tuple(int(i) for i in torch.nonzero(off == off.max())[0])}: got {g.flatten()[off.argmax()]:.9g}, want {want.flatten()[off.argmax()]:.9g} +- {bound.expand_as(want).flatten()[off.argmax()]:.3g}"
