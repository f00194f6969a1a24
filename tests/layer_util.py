"""Plain 64-bit forms of the dense operators and the inputs that their tests share."""
import math

import torch

F64 = torch.float64
ULP32 = 2.0 ** -24          # half a unit in the last place of fp32, relative
ULP16 = 2.0 ** -9           # the same of bf16


def norm_forward(x, gamma, beta, eps):
    x = x.to(F64)
    mu = x.mean(1, keepdim=True)
    rs = 1.0 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    z = (x - mu) * rs
    return z * gamma.to(F64) + beta.to(F64), mu, rs, z


def norm_backward(dy, x, gamma, eps):
    _, _, rs, z = norm_forward(x, gamma, torch.zeros_like(gamma), eps)
    dy = dy.to(F64)
    g = dy * gamma.to(F64)
    dx = rs * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    return dx, (dy * z).sum(0), dy.sum(0)


def gate_weights(value, sigmoid):
    """Weights of the chosen values [T, K], the largest first."""
    if sigmoid:
        # sigma(v) up to a common factor exp(m), m = min(max v, 0): the ratios survive where sigma underflows
        m = value[:, :1].clamp(max=0.0)
        score = torch.where(value > 0, torch.sigmoid(value), torch.exp(value - m) / (1 + torch.exp(value.clamp(max=0.0))))
    else:
        score = torch.exp(value - value[:, :1])
    w = score / score.sum(1, keepdim=True)
    return torch.where(value[:, :1] == -math.inf, torch.zeros_like(w), w)


def gate_forward(logits, K, sigmoid):
    """ids by (value descending, id ascending), NaN above everything; weights over the chosen."""
    value, ids = torch.sort(logits.to(F64), dim=1, descending=True, stable=True)
    value, ids = value[:, :K], ids[:, :K]
    return ids, gate_weights(value, sigmoid), value


def gate_backward(g, logits, ids, w, sigmoid):
    g, w = g.to(F64), w.to(F64)
    d = w * (g - (g * w).sum(1, keepdim=True))
    if sigmoid:
        d = d * torch.sigmoid(-logits.to(F64).gather(1, ids))
    return torch.zeros(logits.shape, dtype=F64, device=logits.device).scatter_(1, ids, d)


def ffn_forward(rows, ranges, w_gate_up, w_down):
    """ranges: [(first, last, expert)]; rows outside stay 0.  Returns out, act, pre."""
    F = w_down.shape[2]
    P, H = rows.shape
    out = torch.zeros((P, H), dtype=F64, device=rows.device)
    act = torch.zeros((P, F), dtype=F64, device=rows.device)
    pre = torch.zeros((P, 2 * F), dtype=F64, device=rows.device)
    for a, b, e in ranges:
        pre[a:b] = rows[a:b].to(F64) @ w_gate_up[e].to(F64).t()
        g, u = pre[a:b, :F], pre[a:b, F:]
        act[a:b] = g * torch.sigmoid(g) * u
        out[a:b] = act[a:b] @ w_down[e].to(F64).t()
    return out, act, pre


def ffn_backward(dy, rows, ranges, w_gate_up, w_down):
    F = w_down.shape[2]
    _, act, pre = ffn_forward(rows, ranges, w_gate_up, w_down)
    dx = torch.zeros(rows.shape, dtype=F64, device=rows.device)
    d_pre, d_act = torch.zeros_like(pre), torch.zeros_like(act)
    dgu, ddn = torch.zeros(w_gate_up.shape, dtype=F64, device=rows.device), torch.zeros(w_down.shape, dtype=F64, device=rows.device)
    for a, b, e in ranges:
        g, u, s = pre[a:b, :F], pre[a:b, F:], torch.sigmoid(pre[a:b, :F])
        d_act[a:b] = dy[a:b].to(F64) @ w_down[e].to(F64)
        d_pre[a:b, :F] = d_act[a:b] * u * s * (1 + g * (1 - s))
        d_pre[a:b, F:] = d_act[a:b] * g * s
        dx[a:b] = d_pre[a:b] @ w_gate_up[e].to(F64)
        dgu[e] += d_pre[a:b].t() @ rows[a:b].to(F64)
        ddn[e] += dy[a:b].to(F64).t() @ act[a:b]
    return dict(dx=dx, dgu=dgu, ddn=ddn, act=act, pre=pre, d_act=d_act, d_pre=d_pre)


def decode_pre(codes):
    """Values of the saved pre-activations: one sign, six exponent (bias 31) and nine mantissa bits."""
    c = codes.view(torch.int16).to(torch.int64) & 0xFFFF
    sign, e, m = 1.0 - 2.0 * (c >> 15), (c >> 9) & 63, (c & 511).to(F64)
    value = torch.where(e > 0, torch.exp2((e - 31).to(F64)) * (1 + m / 512), 2.0 ** -30 * m / 512)
    return torch.where(e == 63, torch.full_like(value, math.nan), sign * value)


def philox_words(counter, key):
    """Philox-4x32-10 on Python integers: the four words of one counter (c0..c3) under key (k0, k1)."""
    c, k, low = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def dropout_keep(n, p, seed, first_block=0):
    """The mask of elements first_block * 8 .. of a call (list of 0/1), and the scale."""
    threshold = int(math.floor(p * 65536.0 + 0.5))
    keep = []
    for b in range(first_block, first_block + (n + 7) // 8):
        words = philox_words((b & 0xFFFFFFFF, b >> 32, 0, 0), (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
        for w in words:
            keep += [int((w & 0xFFFF) >= threshold), int((w >> 16) >= threshold)]
    return keep[:n], (65536.0 / (65536 - threshold) if threshold < 65536 else 0.0)
