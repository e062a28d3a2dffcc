// act_math.cuh -- activations and their slopes in fp32, for the kernels that
// apply them ahead of a rounding to BF16 (the gated MLP of section "Model
// architecture and pretraining system", and linears with an activation).
#pragma once

#include <cstdint>
#include <type_traits>

#include "internal.h"
#include "ptx.cuh"

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

// sigmoid(u) = s and sigmoid(-u) = c from t = e^-|u|, so that neither
// overflows or loses its small values (below |u| = 87; t is zero beyond).
struct Sigmoid {
    float s, c;
};
PURO_DEV Sigmoid sigmoid_both(float u) {
    const float t = ex2_approx(fabsf(u) * -1.44269504f);
    const float r = rcp_approx(1.0f + t), tr = t * r;
    return u >= 0.0f ? Sigmoid{r, tr} : Sigmoid{tr, r};
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

// The activation a and its slope d.  The product z * (a bell around zero) takes
// a bounded z, so that infinities have the slopes 0 and 1.
struct ActSlope {
    float a, d;
};
template <int ACT>
PURO_DEV ActSlope act_slope_f32(float z) {
    const float zb = fminf(fmaxf(z, -128.0f), 128.0f);
    if constexpr (ACT == PURO_ACT_RELU) return ActSlope{z < 0.0f ? 0.0f : z, z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z)};
    if constexpr (ACT == PURO_ACT_SILU) {
        const Sigmoid g = sigmoid_both(z);
        return ActSlope{z * g.s, fmaf(zb * g.s, g.c, g.s)};
    }
    if constexpr (ACT == PURO_ACT_GELU) {
        const Normal n = normal_both(z);  // d = Phi + z e^(-z^2/2) / sqrt(2 pi)
        return ActSlope{z * n.cdf, fmaf(zb * 0.39894228f, n.bell, n.cdf)};
    }
    if constexpr (ACT == PURO_ACT_GELU_TANH) {
        const Sigmoid g = sigmoid_both(z * fmaf(kGeluK, z * z, kGeluC));
        return ActSlope{z * g.s, fmaf(zb * g.s * g.c, fmaf(3.0f * kGeluK, zb * zb, kGeluC), g.s)};
    }
    return ActSlope{z, 1.0f};
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
