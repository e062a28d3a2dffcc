"""64-bit references of the position rotation without a norm: the fraction of a
turn from Python integers, cosines and sines of it in double."""
import math

import torch

import _layer_ops as L


def frequencies(rot, base, scaling="none", factor=1.0, trained=0, fast=32.0, slow=1.0):
    """w_i as doubles, from the definition."""
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    v = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in v]
    if scaling in ("none", "base"):
        return v
    if scaling == "turns":
        keep = [(trained * x / (2 * math.pi) - slow) / (fast - slow) for x in v]
    else:
        at = lambda turns: next_pair(rot, base, trained, turns)  # noqa: E731
        lo, hi = max(0, math.floor(at(fast))), min(rot // 2 - 1, math.ceil(at(slow)))
        keep = [1 - (i - lo) / max(hi - lo, 0.001) for i in range(rot // 2)]
    keep = [min(1.0, max(0.0, k)) for k in keep]
    return [(1 - k) * x / factor + k * x for k, x in zip(keep, v)]


def next_pair(rot, base, trained, turns):
    """The (real) pair whose angle makes `turns` turns over the trained context: base^(-2i/rot) trained = 2 pi turns."""
    return rot / 2 * math.log(trained / (2 * math.pi * turns), base)


def cos_sin(freq, positions, scale=1.0):
    """Tables in double of integer frequencies (2^64ths of a turn) at integer positions."""
    f = [int(x) % 2 ** 64 for x in freq.tolist()]
    turns = torch.tensor([[((p * x) % 2 ** 64) / 2 ** 64 for x in f] for p in positions], dtype=torch.float64)
    turns = turns.reshape(len(positions), len(f))
    return scale * torch.cos(2 * math.pi * turns), scale * torch.sin(2 * math.pi * turns)


def rotation(x, freq, positions, inter, scale=1.0, back=False):
    """y in double of x [T, H, D], and the magnitude that its roundings are relative to; padding rows are zero."""
    at = [max(int(p), 0) for p in positions]
    c, s = cos_sin(freq, at, scale)
    rot = 2 * len(freq)
    y, mag = x.double(), x.double().abs()
    y[..., :rot], mag[..., :rot] = L.rotate(x.double()[..., :rot], c, s, inter, back), L.magnitude(x.double()[..., :rot], c, s, inter)
    # what an angle that is a little off turns into the other channel of the pair
    swapped = L.magnitude(x.double()[..., :rot], torch.full_like(c, abs(scale)), torch.full_like(c, abs(scale)), inter)
    off = torch.zeros_like(y)
    off[..., :rot] = swapped
    pad = torch.tensor([int(p) < 0 for p in positions], dtype=torch.bool)
    for t in (y, mag, off):
        t[pad] = 0
    return y, mag, off
