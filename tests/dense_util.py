"""Plain 64-bit forms of the operators on token rows (8-bit rows, root-mean-square norm, linear) that their tests share."""
import math

import torch

F64 = torch.float64
U = 2.0 ** -24                       # half a unit of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}      # half a step of a result, relative
LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def groups_of(H, group):
    return [(a, min(a + group, H)) for a in range(0, H, group)] if group else [(0, H)]


def nearest_code(u, code):
    """The code nearest to u (float64), halves to even, as a float64 value."""
    if code == torch.int8:
        return torch.round(u)
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(u / step) * step


def pack(x, code, group):
    """(codes as float64, scales float64 [T, groups]) by the definition; a group with a NaN or an infinity: codes 0, scale NaN."""
    x = x.to(F64)
    q, scales = torch.zeros_like(x), []
    for a, b in groups_of(x.shape[1], group):
        part = x[:, a:b]
        most = part.abs().amax(1, keepdim=True)
        good = torch.isfinite(part).all(1, keepdim=True) & (most > 0)
        u = torch.where(good, part * LARGEST[code] / torch.where(good, most, torch.ones_like(most)), torch.zeros_like(part))
        q[:, a:b] = nearest_code(u, code)
        finite = torch.isfinite(part).all(1, keepdim=True)
        scales.append(torch.where(finite, most / LARGEST[code], torch.full_like(most, math.nan)))
    return q, torch.cat(scales, 1)


def values(q, scales, group):
    out = q.to(F64).clone()
    for i, (a, b) in enumerate(groups_of(q.shape[1], group)):
        out[:, a:b] *= scales.to(F64)[:, i:i + 1]
    return out


def rms_forward(s, gamma, eps):
    s = s.to(F64)
    rstd = 1.0 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s * rstd * gamma.to(F64), rstd


def rms_backward(dy, s, gamma, rstd, dsum=None):
    dy, z = dy.to(F64), s.to(F64) * rstd
    g = dy * gamma.to(F64)
    dx = rstd * (g - z * (g * z).mean(1, keepdim=True))
    return dx if dsum is None else dx + dsum.to(F64), (dy * z).sum(0)


def act(v, kind):
    if kind == "relu":
        return v.clamp_min(0)
    if kind == "silu":
        return v * torch.sigmoid(v)
    return 0.5 * v * (1 + torch.erf(v / math.sqrt(2))) if kind == "gelu" else v


def act_slope(v, kind):
    if kind == "relu":
        return (v > 0).to(v.dtype)
    if kind == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(v / math.sqrt(2))) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(v)
