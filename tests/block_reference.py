"""Plain 64-bit restatements of the residual block's operators (torch on the CPU, gradients by autograd)."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # largest relative error of one rounding
KINDS = ("none", "rms", "layer")


def d64(t):
    return None if t is None else t.detach().double().cpu()


def unit(v, kind, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v / ((v * v).mean(1, keepdim=True) + eps).sqrt()


def block_norm(params, x, y, gate, *, pre, post, act, per_gate, eps):
    """(x_out, u); params [3 or 5, d]."""
    bias = params.shape[0] == 5
    if y is not None:
        z = unit(y, post, eps) * params[1]
        if bias:
            z = z + params[4]
        if act != "none":
            g = gate[torch.arange(x.shape[0]) // per_gate]
            z = z * (g if act == "linear" else torch.sigmoid(g))
        x = x + params[2] * z
    u = unit(x, pre, eps) * params[0]
    return x, u + params[3] if bias else u


def activation(v, kind):
    if kind == "relu":
        return v.clamp(min=0)
    if kind == "silu":
        return v * torch.sigmoid(v)
    return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))


def checkpoint(z, cols):
    """The 8-bit format, step by step in fp32 as the header defines it: (q, scales) of z [rows, parts * cols]."""
    z = z.float().cpu()
    q, scales = torch.zeros(z.shape, dtype=torch.int8), []
    for p in range(0, z.shape[1], cols):
        for a in range(p, p + cols, 128):
            g = z[:, a:min(a + 128, p + cols)]
            top = g.abs().amax(1, keepdim=True)
            some = (top >= 1e-30) & torch.isfinite(top)
            inv = torch.where(some, torch.reciprocal(torch.where(some, top, torch.ones_like(top))) * 127.0, torch.zeros_like(top))
            q[:, a:a + g.shape[1]] = torch.where(some, torch.round(g * inv), torch.zeros_like(g)).to(torch.int8)
            scale = torch.where(some, top * torch.tensor(1.0 / 127.0), torch.zeros_like(top))
            scales.append(torch.where(torch.isfinite(top), scale, torch.full_like(top, float("nan"))))
    return q, torch.cat(scales, 1)


def restored(q, scales, cols):
    z = q.double().cpu().clone()
    i = 0
    for p in range(0, z.shape[1], cols):
        for a in range(p, p + cols, 128):
            z[:, a:min(a + 128, p + cols)] *= scales[:, i:i + 1].double().cpu()
            i += 1
    return z


def hidden(z, cols, kind, gated):
    return activation(z[:, :cols], kind) * z[:, cols:] if gated else activation(z, kind)


def close(got, want, dtype, slack, scale=None):
    """Largest excess of |got - want| over one rounding to `dtype` plus slack * scale (scale: of each element, default
    its row's root mean square)."""
    got = got.detach().double().cpu()
    if scale is None:
        scale = want.pow(2).mean(-1, keepdim=True).sqrt()
    unit16 = 0.0 if dtype == torch.float32 else UNIT[dtype]
    tiny = {torch.float16: 2.0 ** -25}.get(dtype, 0.0)          # spacing of the smallest half-precision numbers
    return float(((got - want).abs() - unit16 * want.abs() * (1 + 1e-3) - tiny - slack * scale).max()) if want.numel() else 0.0
