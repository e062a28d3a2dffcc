"""Activations and their slopes over the whole range of BF16 arguments, against 64 bits and relative to their values
(test_gpu_act_backward.py and test_gpu_linear_epilogue.py bound them absolutely, which says nothing of a tail)."""
import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P

DEV, BF = "cuda", torch.bfloat16
CODE = dict(zip(L.ACTS, (P.ACT_NONE, P.ACT_RELU, P.ACT_SILU, P.ACT_GELU, P.ACT_GELU_TANH)))
KINDS = ("silu", "gelu_tanh", "gelu")

# Before the rounding to BF16, relative to the value (for a slope: to the magnitudes of its two terms).  The exponent v of
# e^-u = 2^v is at most 141 where a result is not zero in BF16, and it is off by at most
# SiLU: 2^-18 (the rounding of v - 15, below 128) and 141 * 2^-25 (log2 e): e^-u by 0.69 * 8.0e-6, with ex2 and rcp (2^-22
#       each) and two roundings below 6.2e-6 < 2^-17;
# tanh GELU: 141 * (3 roundings of 2^-24, constants of 2^-24) and 2^-18: 0.69 * 3.8e-5 and those, below 2^-15.
# GELU: Phi's tail by 2^-17.9; e^(-z^2/2) = 2^v by 0.69 * (130 * (2^-24 of z^2 + 2^-25 of the constant) + 2^-18), the
#       polynomial and products 16 * 2^-24: below 2^-15.
# A slope has one product more of each, and tanh GELU's u' its roundings: twice as much.
REL = {"silu": 2.0 ** -17, "gelu_tanh": 2.0 ** -15, "gelu": 2.0 ** -15}
# Absolutely: half a step of a BF16 subnormal, 2^-134, and FP32's subnormals (2^-150, times a factor of at most 128).  A
# sigmoid below 2^-141 is zero: less than half such a step of SiLU (|z| < 2^6.7), of its slope and of tanh GELU (|z| <
# 2^3.4), but not of tanh GELU's slope (|z u'| < 2^8.1).  GELU's bell below 2^-130 is zero, from z = -13.43 on: GELU is
# below 2^-131.3 there and its slope below 2^-127.5, so both may be zero for a subnormal.
SUB = 2.0 ** -142
TINY = {"silu": 2.0 ** -134 + SUB, "gelu_tanh": 2.0 ** -134 + SUB, "gelu": 2.0 ** -131.3 + SUB}
TINY_SLOPE = {"silu": 2.0 ** -134 + SUB, "gelu_tanh": 2.0 ** -132.9 + SUB, "gelu": 2.0 ** -127.5 + SUB}


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _every_finite_value():
    z = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(BF)
    return z[torch.isfinite(z)].view(-1, 16)


def _check(got, ref, size, rel, tiny):
    """Half a BF16 step (2^-8 of the value) and the error before the rounding."""
    err = rel * size
    bad = (got.double() - ref).abs() > 2.0 ** -8 * (ref.abs() + err) + err + tiny
    assert not bool(bad.any()), (f"{int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: "
                                 f"{float(got[bad][0])} for {float(ref[bad][0])}")


def _gate_by_one(z):
    """x, w of a gated product whose gate is z exactly and whose up is 1."""
    m, n = z.shape
    x = torch.cat([z, torch.ones(m, 8, dtype=BF, device=DEV)], 1)
    w = torch.zeros(2 * n, n + 8, dtype=BF, device=DEV)
    w[:n, :n] = torch.eye(n, dtype=BF, device=DEV)
    w[n:, n] = 1
    return x, w


@pytest.mark.gpu
@pytest.mark.parametrize("m", [4080, 16])  # the GEMM's epilogue, the form for a few tokens
@pytest.mark.parametrize("kind", KINDS)
def test_activation_relative_to_its_value(kind, m):
    _need_gpu()
    z = _every_finite_value().view(m, -1)
    eye = torch.eye(z.shape[1], dtype=BF, device=DEV)
    ref, y, h = L.act(z.double(), kind), torch.empty_like(z), torch.empty_like(z)
    P.puro_bf16_linear_fprop_epilogue(z, eye, y, None, CODE[kind])
    _check(y, ref, ref.abs(), REL[kind], TINY[kind])
    P.puro_bf16_gated_fprop(*_gate_by_one(z), CODE[kind], None, h)
    _check(h, ref, ref.abs(), REL[kind], TINY[kind])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_slope_relative_to_its_terms(kind):
    """dz of dy = 1, and [dgate, dup] of dh = up = 1."""
    _need_gpu()
    z = _every_finite_value()
    one, dz, out = torch.ones_like(z), torch.empty_like(z), torch.empty(z.shape[0], 32, dtype=BF, device=DEV)
    zd = z.double()
    d, a = L.slope(zd, kind), L.act(zd, kind)
    first = (a / zd).where(zd != 0, torch.full_like(zd, 0.5))  # the sigmoid, or Phi
    size = first + (d - first).abs()
    P.puro_act_backward_bf16(one, z, CODE[kind], dz, None)
    _check(dz, d, size, 2 * REL[kind], TINY_SLOPE[kind])
    P.puro_gated_backward_bf16(one, z, one, CODE[kind], out)
    _check(out[:, :16], d, size, 2 * REL[kind], TINY_SLOPE[kind])
    _check(out[:, 16:], a, a.abs(), REL[kind], TINY[kind])


@pytest.mark.gpu
def test_gated_form_and_separate_swiglu_agree():
    """h of the gated product and h of puro_swiglu_bf16 of the same gate and up: a BF16 step apart at most."""
    _need_gpu()
    z = _every_finite_value()
    h, sep = torch.empty_like(z), torch.empty_like(z)
    P.puro_bf16_gated_fprop(*_gate_by_one(z), P.ACT_SILU, None, h)
    P.puro_swiglu_bf16(z, torch.ones_like(z), sep)
    assert bool(((h.double() - sep.double()).abs() <= 2.0 ** -7 * sep.double().abs() + 2.0 ** -133).all())
