// act_math.cuh -- activations and their slopes in fp32, for the kernels that
// apply them ahead of a rounding to BF16 (the gated MLP of section "Model
// architecture and pretraining system", and linears with an activation).
#pragma once

#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>

#include "internal.h"
#include "ptx.cuh"
#include "quant_math.cuh"

namespace puro {

// 2^x and 1/x by the special-function unit (PTX ex2.approx / rcp.approx:
// relative error around 2^-22; subnormal results flush to zero).
PURO_DEV float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
PURO_DEV float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The normal distribution function Phi(z) and its bell.  Phi(-x) e^(x^2/2), x >= 0 (Mills'
// ratio over sqrt(2 pi)), falls off as 1 / x, so it is t P(t), t = 1 / (1 + p x), P a polynomial
// of degree 6.  p and P have the least maximum over 0 <= x <= 14 of the error of Phi(-x) over
// min(7.5e-8, 2^-16 Phi(-x)), found by linear programming on a grid: 2.0e-8 and, in the tail,
// 2^-17.9 of its value; with the FP32 roundings 2.2e-7 and 2^-17.  The bell is taken 16 times as
// large, which costs no rounding near zero and keeps every normal GELU and slope (it is zero below
// z = -13.4).  Formula 7.1.26 of Abramowitz and Stegun's Handbook, two terms shorter, bounds the
// absolute error alone (1.5e-7 of erf): 0.16% off at -5, 2% at -10.  CUDA's normcdff, which holds
// the tail too, made the GEMM's epilogue its bound: [8192, 2048] x 6144 84.9 us.  Slopes take it
// one value at a time (two an instruction, of the shorter formula: 76.6 us for 74.0 on [8192, 8960]).
constexpr float kBell = 16.0f, kBellLog2 = 4.0f;
constexpr float kMillsP = 0.255f;
constexpr float kMills0 = 0.1013295054f / kBell, kMills1 = 0.1078548532f / kBell, kMills2 = 0.0569961062f / kBell, kMills3 = 0.2068689727f / kBell,
                kMills4 = -0.1678357881f / kBell, kMills5 = 0.2753503274f / kBell, kMills6 = -0.0805639588f / kBell;
struct Normal {
    float cdf, bell;  // Phi(z), kBell e^(-z^2/2)
};
PURO_DEV Normal normal_both(float z) {
    const float t = rcp_approx(fmaf(fabsf(z), kMillsP, 1.0f));
    const float e = ex2_approx(fmaf(z * z, -0.72134752f, kBellLog2));
    float q = fmaf(t, kMills6, kMills5);
    q = fmaf(t, q, kMills4);
    q = fmaf(t, q, kMills3);
    q = fmaf(t, q, kMills2);
    q = fmaf(t, q, kMills1);
    q = fmaf(t, q, kMills0);
    q = t * q * e;
    return Normal{z >= 0.0f ? 1.0f - q : q, e};
}

constexpr float kGeluC = 1.5957691216f;              // 2 sqrt(2 / pi)
constexpr float kGeluK = 0.044715f * 1.5957691216f;  // gelu_tanh(z) = z sigmoid(z (kGeluC + kGeluK z^2))

PURO_DEV uint64_t splat(float x) { return f32x2(x, x); }
PURO_DEV uint64_t widen2(uint32_t w) { return f32x2(bf16_lo(w), bf16_hi(w)); }
// Both BF16 values kept within 128 of zero (NaN stays).
PURO_DEV uint32_t bounded2(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b32 t;\n\tmin.NaN.bf16x2 t, %1, %2;\n\tmax.NaN.bf16x2 %0, t, %3;\n\t}" : "=r"(r) : "r"(w), "r"(0x43004300u), "r"(0xC300C300u));
    return r;
}

// sigmoid(u) = 1 / (1 + 2^v), v = -u log2 e, two at a time, from v - 15: 2^15 sigmoid =
// 1 / (2^-15 + 2^(v - 15)), so that neither the power nor the reciprocal leaves the normal
// range before v = 141, where |z| sigmoid is below half of BF16's last subnormal (unscaled
// they do from v = 126 on: SiLU of -88 came out as 0 for -5.3e-37).  The exact scaling by
// 2^-15 gives subnormals too; beyond, the sigmoid is zero.  The rounding of v - 15 costs at
// most 2^-21.5 of the sigmoid above z = -4.8.
constexpr float kSigmoidShift = 15.0f, kSigmoidScale = 0x1p-15f;
PURO_DEV uint64_t sigmoid2(uint64_t v_less_shift) {
    float lo, hi;
    split_f32x2(v_less_shift, lo, hi);
    split_f32x2(add_f32x2(f32x2(ex2_approx(lo), ex2_approx(hi)), splat(kSigmoidScale)), lo, hi);
    return mul_f32x2(f32x2(rcp_approx(lo), rcp_approx(hi)), splat(kSigmoidScale));
}
PURO_DEV uint64_t silu_exponent2(uint64_t z) {  // v - 15, u = z
    return fma_f32x2(z, splat(-1.44269504f), splat(-kSigmoidShift));
}
PURO_DEV uint64_t tanh_gelu_exponent2(uint64_t z) {  // v - 15, u = z (kGeluC + kGeluK z^2)
    const uint64_t f = fma_f32x2(mul_f32x2(z, z), splat(-1.44269504f * kGeluK), splat(-1.44269504f * kGeluC));
    return fma_f32x2(z, f, splat(-kSigmoidShift));
}

// -|x| but at least -64, and max(x, 0); NaN stays.
PURO_DEV float neg_abs_bounded(float x) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(-fabsf(x)), "f"(-64.0f));
    return r;
}
PURO_DEV float relu_nan(float x) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(0.0f));
    return r;
}

// The activations of two FP32 values, two an instruction.  GELU as max(z, 0) - |z| q, q =
// Phi(-|z|) as in normal_both (beyond 64 q is zero, so infinities have their limits).
template <int ACT>
PURO_DEV uint64_t act_pair(uint64_t z) {
    if constexpr (ACT == PURO_ACT_SILU) return mul_f32x2(z, sigmoid2(silu_exponent2(z)));
    if constexpr (ACT == PURO_ACT_GELU_TANH) return mul_f32x2(z, sigmoid2(tanh_gelu_exponent2(z)));
    if constexpr (ACT == PURO_ACT_RELU || ACT == PURO_ACT_GELU) {
        float a, b, lo, hi;
        split_f32x2(z, a, b);
        const uint64_t pos = f32x2(relu_nan(a), relu_nan(b));
        if constexpr (ACT == PURO_ACT_RELU) return pos;
        const uint64_t n = f32x2(neg_abs_bounded(a), neg_abs_bounded(b));
        split_f32x2(fma_f32x2(n, splat(-kMillsP), splat(1.0f)), lo, hi);
        const uint64_t t = f32x2(rcp_approx(lo), rcp_approx(hi));
        split_f32x2(fma_f32x2(mul_f32x2(n, n), splat(-0.72134752f), splat(kBellLog2)), lo, hi);
        const uint64_t e = f32x2(ex2_approx(lo), ex2_approx(hi));
        uint64_t q = fma_f32x2(t, splat(kMills6), splat(kMills5));
        q = fma_f32x2(t, q, splat(kMills4));
        q = fma_f32x2(t, q, splat(kMills3));
        q = fma_f32x2(t, q, splat(kMills2));
        q = fma_f32x2(t, q, splat(kMills1));
        q = fma_f32x2(t, q, splat(kMills0));
        return fma_f32x2(mul_f32x2(n, mul_f32x2(t, q)), e, pos);
    }
    return z;
}

// Activations of a BF16 pair, and their slopes, in packed arithmetic.  With s =
// sigmoid(u), Phi the normal distribution function:
//   SiLU (u = z):  a = z s,    d = s + z s (1 - s)
//   tanh GELU:     a = z s,    d = s + z s (1 - s) u'
//   GELU:          a = z Phi,  d = Phi + z e^(-z^2/2) / sqrt(2 pi)
// Slopes take z within 128 of zero, beyond which they are 0 and 1 to the last bit:
// infinities then have those slopes too.  1 - s is taken as a difference: 6e-8 off
// where s is near 1, where d is too.
template <int ACT>
PURO_DEV uint64_t act2(uint32_t w) {
    return act_pair<ACT>(widen2(w));
}
template <int ACT>
PURO_DEV uint64_t slope2(uint32_t w) {
    if constexpr (ACT == PURO_ACT_NONE) return splat(1.0f);
    if constexpr (ACT == PURO_ACT_RELU) {
        auto step = [](float x) { return x > 0.0f ? 1.0f : (x <= 0.0f ? 0.0f : x); };
        return f32x2(step(bf16_lo(w)), step(bf16_hi(w)));
    }
    const uint32_t wb = bounded2(w);
    const uint64_t z = widen2(wb);
    if constexpr (ACT == PURO_ACT_GELU) {
        const Normal n0 = normal_both(bf16_lo(wb)), n1 = normal_both(bf16_hi(wb));
        return fma_f32x2(mul_f32x2(z, splat(0.39894228f / kBell)), f32x2(n0.bell, n1.bell), f32x2(n0.cdf, n1.cdf));
    }
    constexpr bool kTanh = ACT == PURO_ACT_GELU_TANH;
    const uint64_t s = sigmoid2(kTanh ? tanh_gelu_exponent2(z) : silu_exponent2(z));
    uint64_t bell = mul_f32x2(mul_f32x2(z, s), fma_f32x2(s, splat(-1.0f), splat(1.0f)));
    if constexpr (kTanh) bell = mul_f32x2(bell, fma_f32x2(mul_f32x2(z, z), splat(3.0f * kGeluK), splat(kGeluC)));
    return add_f32x2(bell, s);
}

PURO_DEV uint32_t pack_bf16x2(uint64_t v) {
    float lo, hi;
    split_f32x2(v, lo, hi);
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}

// The activation of z (puro_act_t).
template <int ACT>
PURO_DEV float act_f32(float z) {
    float lo, hi;
    split_f32x2(act_pair<ACT>(f32x2(z, 0.0f)), lo, hi);
    return lo;
}

// dz = dy * act'(z) of two BF16 pairs; the unrounded values are added to s0, s1.
template <int ACT>
PURO_DEV uint32_t act_backward2(uint32_t dy, uint32_t z, float &s0, float &s1) {
    const uint64_t d = ACT == PURO_ACT_NONE ? widen2(dy) : mul_f32x2(widen2(dy), slope2<ACT>(z));
    float lo, hi;
    split_f32x2(d, lo, hi);
    s0 += lo;
    s1 += hi;
    return pack_bf16x2(d);
}

// dgate = dh * (up * act'(gate)) and dup = dh * act(gate) of two BF16 pairs.
template <int ACT>
PURO_DEV uint32_t gate_backward2(uint32_t dh, uint32_t gate, uint32_t up) {
    return pack_bf16x2(mul_f32x2(widen2(dh), mul_f32x2(widen2(up), slope2<ACT>(gate))));
}
template <int ACT>
PURO_DEV uint32_t up_backward2(uint32_t dh, uint32_t gate) {
    return pack_bf16x2(mul_f32x2(widen2(dh), act2<ACT>(gate)));
}

// f(std::integral_constant<int, act>): one copy of the code for each activation.
template <class F>
PURO_DEV void act_dispatch(int act, F f) {
    switch (act) {
        case PURO_ACT_RELU: return f(std::integral_constant<int, PURO_ACT_RELU>{});
        case PURO_ACT_SILU: return f(std::integral_constant<int, PURO_ACT_SILU>{});
        case PURO_ACT_GELU: return f(std::integral_constant<int, PURO_ACT_GELU>{});
        case PURO_ACT_GELU_TANH: return f(std::integral_constant<int, PURO_ACT_GELU_TANH>{});
        default: return f(std::integral_constant<int, PURO_ACT_NONE>{});
    }
}

}  // namespace puro
