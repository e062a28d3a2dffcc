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


def exact(v, steps=STEPS, kept=1.0):
    """kept: what sums over X's rows leave of themselves."""
    v = v.double()
    tall = v.shape[0] > v.shape[1]
    x = v.T if tall else v
    norm = x.norm()
    x = x / norm if norm > 0 else x
    for a, b, c in steps:
        g = kept * (x @ x.T)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def _half(x, scale):
    return (x * scale).to(torch.float16).double() / scale


def _scale(most):
    return 2.0 ** 14 if most <= 0 else 2.0 ** min(100, math.floor(math.log2(32768 / (most * (1 + 1 / 64)))))


PRECISE, LONG = 32, 512  # up to so many rows every number is kept as two FP16 ones; the Gram matrix of longer rows is of their upper halves


def model(v, steps=STEPS):
    v = v.double()
    tall = v.shape[0] > v.shape[1]
    x = v.T if tall else v
    norm = x.norm()
    x = x / norm if norm > 0 else x
    eye = torch.eye(len(x), dtype=torch.float64)
    every = len(x) <= PRECISE
    most, i = 1.0, 0

    def bounds(step, most):
        s = torch.linspace(0, most, 4097, dtype=torch.float64)
        a, b, c = step
        p = (a + b * s ** 2 + c * s ** 4).abs()
        return float(p.max()), float((s * p).max()) * (1 + 1 / 64)

    def keep(x, scale, lo=False):
        """hi and lo of a result."""
        hi = _half(x, scale)
        return hi, _half(x - hi, scale) if lo or every else 0 * x

    def times(x, y):
        return x[0] @ y[0] + x[0] @ y[1] + (x[1] @ y[0] if every else 0)

    def turn(x):
        return x[0].T, x[1].T

    def mirror(x):
        return tuple(torch.triu(h) + torch.triu(h, 1).T for h in x)

    sx = 2.0 ** 14
    while i < len(steps):
        pair = i + 1 < len(steps)
        x = keep(x, sx, pair and i == 0)
        a, b, c = steps[i]
        mp, out = bounds(steps[i], most)
        gram = times(x, turn(x)) if every and x[0].shape[1] <= LONG else x[0] @ x[0].T
        g = keep(gram, _scale(most ** 2), pair and i > 0)
        low = g if every else (g[0], 0 * g[0])  # elsewhere G's lo is for T alone
        b0 = keep(a * eye + b * (low[0] + low[1]) + c * times(low, low), _scale(mp))
        if pair:
            a, b, c = steps[i + 1]
            mp1, out1 = bounds(steps[i + 1], out)
            t = keep(times(b0, g), _scale(most ** 2 * mp))
            g = mirror(keep(times(b0, turn(t)), _scale(out ** 2)))
            b1 = keep(a * eye + b * (g[0] + g[1]) + c * times(g, g), _scale(mp1))
            b0, out = keep(times(b1, b0), _scale(mp * mp1)), out1
        x = times(b0, x)
        most, sx = out, _scale(out)
        i += 2 if pair else 1
    return x.T if tall else x


def bound(v, u_type, steps=STEPS):
    """What u may be off by in the 2-norm: twice the model's error, which is one draw of the same roundings; what the model lacks or draws of
    few values may differ by; and half a step of u's type.  The second is 2^-9 (the last product's two FP16 operands are each within 2^-11
    and of norm at most 2 to u's 1), or where every number has 22 digits what FP32's sums add: 2^-22 each, of which the first steps' are
    blown up 3.4445^5 = 485 times, so 2^-13.  Long rows add what their sums in FP32 lose: an entry of G = X X^T is a sum of n products, each
    addition of which may cut off a step, 2^-23 of the sum, all in the same direction; so what u changes by where each G is 1 - n 2^-23 of
    itself."""
    e = exact(v, steps)
    more = 2.0 ** -13 if min(v.shape) <= PRECISE else 2.0 ** -9
    return e, (2 * float((model(v, steps) - e).norm()) + float((exact(v, steps, 1 - max(v.shape) * 2.0 ** -23) - e).norm()) +
               (more + (2.0 ** -8 if u_type == torch.bfloat16 else 2.0 ** -24)) * float(e.norm()))


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
