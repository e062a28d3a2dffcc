"""64-bit CPU references of the decoder layer's steps beside its linears:
query and key norms with rotation, activations and gates, linears with an
epilogue.  Plain torch double arithmetic on the CPU, gradients from their
formulas (which test_layer_ops_reference.py compares with differences)."""
import math

import torch

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def rotate(x, cos, sin, inter, back=False):
    """x [T, H, D]; cos, sin [T, rot / 2]."""
    rot = 2 * cos.shape[1]
    c, s = cos[:, None], -sin[:, None] if back else sin[:, None]
    y = x.clone()
    ia = slice(0, rot, 2) if inter else slice(0, rot // 2)
    ib = slice(1, rot, 2) if inter else slice(rot // 2, rot)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def magnitude(x, cos, sin, inter):
    """|a cos| + |b sin| and |b cos| + |a sin|: what the roundings of a rotation are relative to."""
    rot = 2 * cos.shape[1]
    c, s = cos[:, None].abs(), sin[:, None].abs()
    y = x.abs()
    ia = slice(0, rot, 2) if inter else slice(0, rot // 2)
    ib = slice(1, rot, 2) if inter else slice(rot // 2, rot)
    a, b = y[..., ia].clone(), y[..., ib].clone()
    y[..., ia], y[..., ib] = a * c + b * s, b * c + a * s
    return y


def qk_forward(x, gain, cos, sin, inter, eps):
    """y, rstd, and the magnitude that y's roundings are relative to."""
    rstd = (x.pow(2).mean(-1, keepdim=True) + eps) ** -0.5
    n = x * rstd * (1 if gain is None else gain)
    return rotate(n, cos, sin, inter), rstd[..., 0], magnitude(n, cos, sin, inter)


def qk_backward(dy, x, rstd, gain, cos, sin, inter):
    """dx, dgain, dx's magnitude and the sum of the gain gradient's terms' magnitudes."""
    g = torch.ones(x.shape[-1], dtype=x.dtype) if gain is None else gain
    r = rstd[..., None]
    xh = x * r
    dn = rotate(dy, cos, sin, inter, back=True)
    m = (dn * g * xh).mean(-1, keepdim=True)
    dx = r * (dn * g - xh * m)
    mag = magnitude(dy, cos, sin, inter)
    return dx, (dn * xh).sum((0, 1)), r.abs() * (mag * g.abs() + xh.abs() * (mag * g.abs() * xh.abs()).mean(-1, keepdim=True)), \
        (mag * xh.abs()).sum((0, 1))


def act(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    return z * torch.sigmoid(2 * u)


def slope(z, kind):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = 2 * math.sqrt(2 / math.pi)
    u, du = (z, 1.0) if kind == "silu" else (c * (z + 0.044715 * z ** 3), c * (1 + 3 * 0.044715 * z * z))
    return torch.sigmoid(u) + z * torch.sigmoid(u) * torch.sigmoid(-u) * du


def gated(gate, up, kind):
    return act(gate, kind) * up


def gated_backward(dh, gate, up, kind):
    return dh * up * slope(gate, kind), dh * act(gate, kind)
