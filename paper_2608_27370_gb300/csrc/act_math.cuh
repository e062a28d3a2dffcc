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

// The normal distribution function Phi(z) and e^(-z^2/2), by formula 7.1.26 of
// Abramowitz and Stegun, Handbook of Mathematical Functions (erf to 1.5e-7 by a
// polynomial in 1 / (1 + p x) times e^(-x^2), x = |z| / sqrt(2)); with the FP32
// roundings Phi is within 2^-21.  Behind the GEMM's epilogue CUDA's normcdff
// made it the bound: [8192, 2048] x 6144 84.9 us.
struct Normal {
    float cdf, bell;
};
PURO_DEV Normal normal_both(float z) {
    const float t = rcp_approx(fmaf(fabsf(z), 0.3275911f * 0.70710678f, 1.0f));
    const float e = ex2_approx(z * z * -0.72134752f);
    float q = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
    q = fmaf(t, q, 0.5f * 1.421413741f);
    q = fmaf(t, q, 0.5f * -0.284496736f);
    q = fmaf(t, q, 0.5f * 0.254829592f) * (t * e);
    return Normal{z >= 0.0f ? 1.0f - q : q, e};
}

constexpr float kGeluC = 1.5957691216f;              // 2 sqrt(2 / pi)
constexpr float kGeluK = 0.044715f * 1.5957691216f;  // gelu_tanh(z) = z sigmoid(z (kGeluC + kGeluK z^2))

// The activation of z (puro_act_t).
template <int ACT>
PURO_DEV float act_f32(float z) {
    if constexpr (ACT == PURO_ACT_RELU) return z < 0.0f ? 0.0f : z;  // (NaN stays)
    // (e^-u may overflow: the reciprocal is then zero, and the activation below 1e-36)
    if constexpr (ACT == PURO_ACT_SILU) return z * rcp_approx(1.0f + ex2_approx(z * -1.44269504f));
    if constexpr (ACT == PURO_ACT_GELU) return z * normal_both(z).cdf;
    if constexpr (ACT == PURO_ACT_GELU_TANH)
        return z * rcp_approx(1.0f + ex2_approx(z * fmaf(-1.44269504f * kGeluK, z * z, -1.44269504f * kGeluC)));
    return z;
}

PURO_DEV float bounded(float z) { return fminf(fmaxf(z, -128.0f), 128.0f); }
PURO_DEV uint64_t splat(float x) { return f32x2(x, x); }

// Two activations a and their slopes d, in packed arithmetic.  Where the slope has
// a product z * (a bell around zero) it takes a bounded z, so that infinities have
// the slopes 0 and 1 (NaN stays, through the sigmoid or Phi).  With s = sigmoid(u):
//   SiLU (u = z):      a = z s,  d = s + z s (1 - s)
//   tanh GELU:         a = z s,  d = s + z s (1 - s) u',  u = z (c + k z^2)
//   GELU:              a = z Phi,  d = Phi + z e^(-z^2/2) / sqrt(2 pi)
// 1 - s is taken as a difference: 6e-8 off where s is near 1, where d is too.
struct ActSlope2 {
    uint64_t a, d;
};
template <int ACT>
PURO_DEV ActSlope2 act_slope2(float z0, float z1) {
    const uint64_t z = f32x2(z0, z1);
    if constexpr (ACT == PURO_ACT_RELU) {
        auto relu = [](float x) { return x < 0.0f ? 0.0f : x; };
        auto step = [](float x) { return x > 0.0f ? 1.0f : (x <= 0.0f ? 0.0f : x); };
        return ActSlope2{f32x2(relu(z0), relu(z1)), f32x2(step(z0), step(z1))};
    }
    if constexpr (ACT == PURO_ACT_SILU || ACT == PURO_ACT_GELU_TANH) {
        constexpr bool kTanh = ACT == PURO_ACT_GELU_TANH;
        uint64_t u = mul_f32x2(z, splat(-1.44269504f));  // -u log2 e
        if constexpr (kTanh)
            u = mul_f32x2(z, fma_f32x2(mul_f32x2(z, z), splat(-1.44269504f * kGeluK), splat(-1.44269504f * kGeluC)));
        float lo, hi;
        split_f32x2(u, lo, hi);
        split_f32x2(add_f32x2(f32x2(ex2_approx(lo), ex2_approx(hi)), splat(1.0f)), lo, hi);
        const uint64_t s = f32x2(rcp_approx(lo), rcp_approx(hi));
        const uint64_t zb = f32x2(bounded(z0), bounded(z1));
        uint64_t bell = mul_f32x2(mul_f32x2(zb, s), fma_f32x2(s, splat(-1.0f), splat(1.0f)));
        if constexpr (kTanh) bell = mul_f32x2(bell, fma_f32x2(mul_f32x2(zb, zb), splat(3.0f * kGeluK), splat(kGeluC)));
        return ActSlope2{mul_f32x2(z, s), add_f32x2(bell, s)};
    }
    if constexpr (ACT == PURO_ACT_GELU) {
        const Normal n0 = normal_both(z0), n1 = normal_both(z1);
        const uint64_t cdf = f32x2(n0.cdf, n1.cdf), zb = f32x2(bounded(z0), bounded(z1));
        return ActSlope2{mul_f32x2(z, cdf), fma_f32x2(mul_f32x2(zb, splat(0.39894228f)), f32x2(n0.bell, n1.bell), cdf)};
    }
    return ActSlope2{z, splat(1.0f)};
}

PURO_DEV uint32_t pack_bf16x2(uint64_t v) {
    float lo, hi;
    split_f32x2(v, lo, hi);
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}

// dz = dy * act'(z) of two BF16 pairs; the unrounded values are added to s0, s1.
template <int ACT>
PURO_DEV uint32_t act_backward2(uint32_t dy, uint32_t z, float &s0, float &s1) {
    const uint64_t d = mul_f32x2(f32x2(bf16_lo(dy), bf16_hi(dy)), act_slope2<ACT>(bf16_lo(z), bf16_hi(z)).d);
    float lo, hi;
    split_f32x2(d, lo, hi);
    s0 += lo;
    s1 += hi;
    return pack_bf16x2(d);
}

// dgate = dh * (up * act'(gate)) and dup = dh * act(gate) of two BF16 pairs.
template <int ACT>
PURO_DEV void gated_backward2(uint32_t dh, uint32_t gate, uint32_t up, uint32_t &dgate, uint32_t &dup) {
    const ActSlope2 s = act_slope2<ACT>(bf16_lo(gate), bf16_hi(gate));
    const uint64_t d = f32x2(bf16_lo(dh), bf16_hi(dh));
    dgate = pack_bf16x2(mul_f32x2(d, mul_f32x2(f32x2(bf16_lo(up), bf16_hi(up)), s.d)));
    dup = pack_bf16x2(mul_f32x2(d, s.a));
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
