"""The Muon direction in 64 bits, and a model of the kernels' roundings.

exact() is the definition.  model() takes the steps as the kernels do, two at a
time, and rounds to FP16 where they do, all else in 64 bits: what it is off by is
what FP16 operands cost on these very inputs, so that the kernels' error, another
draw of the same roundings, is of the same size.
"""
import math

import torch

STEPS = ((3.4445, -4.7750, 2.0315),) * 5


def update(g, m, mu, nesterov):
    """The momentum after the gradient, and V."""
    if m is None:
        return None, g
    m = mu * m + g
    return m, g + mu * m if nesterov else m


def exact(v, steps=STEPS):
    v = v.double()
    tall = v.shape[0] > v.shape[1]
    x = v.T if tall else v
    norm = x.norm()
    x = x / norm if norm > 0 else x
    for a, b, c in steps:
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def _half(x, scale):
    return (x * scale).to(torch.float16).double() / scale


def _scale(most):
    return 2.0 ** 14 if most <= 0 else 2.0 ** min(100, math.floor(math.log2(32768 / (most * (1 + 1 / 64)))))


def model(v, steps=STEPS):
    v = v.double()
    tall = v.shape[0] > v.shape[1]
    x = v.T if tall else v
    norm = x.norm()
    x = x / norm if norm > 0 else x
    eye = torch.eye(len(x), dtype=torch.float64)
    most, i = 1.0, 0

    def bounds(step, most):
        s = torch.linspace(0, most, 4097, dtype=torch.float64)
        a, b, c = step
        p = (a + b * s ** 2 + c * s ** 4).abs()
        return float(p.max()), float((s * p).max()) * (1 + 1 / 64)

    sx = 2.0 ** 14
    while i < len(steps):
        hi = _half(x, sx)
        pair = i + 1 < len(steps)
        lo = _half(x - hi, sx) if pair and i == 0 else 0 * x
        a, b, c = steps[i]
        mp, out = bounds(steps[i], most)
        g = _half(hi @ hi.T, _scale(most ** 2))
        b0 = _half(a * eye + b * g + c * (g @ g), _scale(mp))
        if pair:
            a, b, c = steps[i + 1]
            mp1, out1 = bounds(steps[i + 1], out)
            g_lo = _half(hi @ hi.T - g, _scale(most ** 2)) if i else 0 * g
            t = _half(b0 @ (g + g_lo), _scale(most ** 2 * mp))
            g = _half(b0 @ t.T, _scale(out ** 2))
            g = torch.triu(g) + torch.triu(g, 1).T
            b1 = _half(a * eye + b * g + c * (g @ g), _scale(mp1))
            b0, out = _half(b1 @ b0, _scale(mp * mp1)), out1
        x = b0 @ hi + b0 @ lo
        most, sx = out, _scale(out)
        i += 2 if pair else 1
    return x.T if tall else x


def bound(v, u_type, steps=STEPS):
    """What u may be off by in the 2-norm: twice the model's error, which is one draw of the same roundings; 2^-9 for matrices of
    few values, whose draws differ (the last product's two FP16 operands are each within 2^-11 and of norm at most 2 to u's 1); and
    half a step of u's type."""
    e = exact(v, steps)
    return e, 2 * float((model(v, steps) - e).norm()) + (2.0 ** -9 + (2.0 ** -8 if u_type == torch.bfloat16 else 2.0 ** -24)) * float(e.norm())


def gradient(r, c, seed, kind="mixed"):
    """Low rank and noise in all directions, as batches' gradients are; or noise alone."""
    g = torch.Generator().manual_seed(seed)
    k = max(1, min(r, c, 16) // 2)
    noise = torch.randn(r, c, generator=g)
    if kind == "noise":
        return noise * 1e-3
    return (torch.randn(r, k, generator=g) @ torch.randn(k, c, generator=g) / math.sqrt(k) + 0.5 * noise) * 1e-3


def singular_value(s, steps=STEPS):
    """What the steps make of one singular value."""
    for a, b, c in steps:
        s = s * (a + b * s * s + c * s ** 4)
    return s
