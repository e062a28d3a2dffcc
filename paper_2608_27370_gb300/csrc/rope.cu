// rope.cu -- the position rotation of queries and keys without a norm, its
// backward, and tables of its cosines and sines (Puro-2B trains its FP8 path on
// layers of the Qwen2 architecture, whose queries and keys are rotated as the qkv
// projection leaves them).
//
// Pair i of a head turns by the angle p w_i at position p, and is multiplied by a
// scale that long contexts want:
//     (a, b) -> scale (a cos - b sin, b cos + a sin);
// backward with the sines' signs exchanged.
//
// The angle in whole turns is p w_i / (2 pi), of which only the fraction counts.
// So a frequency is kept as the 64-bit integer F_i = w_i / (2 pi) 2^64, and p F_i
// modulo 2^64 is the fraction of a turn in units of 2^-64: an integer product,
// which wraps round where the angle does, loses nothing at far positions, and
// needs neither 64-bit floating point nor tables in memory.  F_i is made in doubles: the
// power's argument, of which w_i is off by |ln w_i| 2^-53, at most four roundings of 2^-53
// more, and the fraction cut off, one unit.  w |ln w| is at most 0.37, so the angle at
// position 2^31 is within 2^-20 (2^-21.6 the worst of 750 tables of all scalings).
#include <cuda_bf16.h>

#include "internal.h"
#include "ptx.cuh"
#include "rotation.cuh"

namespace puro {

constexpr int kRopeThreads = 128;
constexpr int kRopeBatch = 4;  // heads of a token a group loads at once

// The upper 32 bits of the fraction of a turn that p F leaves.
PURO_DEV uint32_t turn_of(uint32_t p, uint64_t f) {
    return __umulhi(p, static_cast<uint32_t>(f)) + p * static_cast<uint32_t>(f >> 32);
}

// Bound by memory: x is read once and y written once, beside 64 bytes of
// frequencies a lane (of the same cache lines for every token).  The angles are
// worked out anew for each batch of heads: two multiplications, a conversion and
// two calls of the special function unit for a pair.  Sines and cosines are within
// 2^-19 (2^-21 of the functions on [-pi, pi], 3 pi 2^-24 of the angle's roundings);
// half a step of the BF16 that follows is 2^-9.
template <int G, bool INTER>
__global__ void __launch_bounds__(kRopeThreads, 8) rope_kernel(const RopeArgs p) {
    constexpr int B = kRopeBatch;
    pdl_wait();
    pdl_launch_dependents();
    const QkLane l = qk_lane(threadIdx.x % G, p.D, p.rot, INTER);
    const unsigned q_batches = (p.q.heads + B - 1) / B, batches = q_batches + (p.k.heads + B - 1) / B;
    const int64_t t = static_cast<int64_t>(blockIdx.x / batches) * (kRopeThreads / G) + threadIdx.x / G;
    const unsigned batch = blockIdx.x % batches;
    const bool is_q = batch < q_batches;
    if (t >= p.tokens || !l.in) return;
    const QkHeads &src = is_q ? p.q : p.k, &dst = is_q ? p.q_out : p.k_out;
    const int h0 = static_cast<int>(is_q ? batch : batch - q_batches) * B, n = min(B, src.heads - h0);
    const uint16_t *from = src.data + t * src.token_stride + h0 * src.head_stride;
    const int64_t pos = p.positions ? __ldg(p.positions + t) : t;
    uint4 x[B][2];  // (y may be x: loaded past L1, where a neighbour's part of a sector would stay as it was)
#pragma unroll
    for (int b = 0; b < B; ++b) {
        x[b][0] = x[b][1] = make_uint4(0, 0, 0, 0);
        if (b < n) {
            x[b][0] = __ldcg(reinterpret_cast<const uint4 *>(from + l.o0));
            x[b][1] = __ldcg(reinterpret_cast<const uint4 *>(from + l.o1));
        }
        from += src.head_stride;
    }
    uint64_t c[4], s[4], m[4];
    if (l.turned) {
        const uint4 *f = reinterpret_cast<const uint4 *>(p.freq + l.pair);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 w = __ldg(f + j);
            float cs[2], sn[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint64_t fk = k ? (static_cast<uint64_t>(w.w) << 32 | w.z) : (static_cast<uint64_t>(w.y) << 32 | w.x);
                // the nearer half turn: [-pi, pi)
                const float a = static_cast<float>(static_cast<int32_t>(turn_of(static_cast<uint32_t>(pos), fk))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
                cs[k] = p.scale * __cosf(a);
                sn[k] = p.sin_scale * __sinf(a);
            }
            c[j] = f32x2(cs[0], cs[1]);
            s[j] = f32x2(sn[0], sn[1]);
            m[j] = f32x2(-sn[0], -sn[1]);
        }
    }
    uint16_t *to = dst.data + t * dst.token_stride + h0 * dst.head_stride;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        if (b >= n) break;
        uint4 y0 = x[b][0], y1 = x[b][1];
        if (l.turned) {
            Pairs v = unpack16<INTER>(y0, y1);
            turn(v, c, s, m);
            pack16<INTER>(v, y0, y1);
        }
        if (pos < 0) y0 = y1 = make_uint4(0, 0, 0, 0);  // padding, whatever the row holds
        *reinterpret_cast<uint4 *>(to + l.o0) = y0;
        *reinterpret_cast<uint4 *>(to + l.o1) = y1;
        to += dst.head_stride;
    }
}

cudaError_t launch_rope(const RopeArgs &p, cudaStream_t s) {
    const int64_t per = kRopeThreads / group_lanes(p.D);
    auto batches = [](int heads) { return (heads + kRopeBatch - 1) / kRopeBatch; };
    const int64_t grid = (p.tokens + per - 1) / per * (batches(p.q.heads) + batches(p.k.heads));
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_pdl(PURO_QK_KERNEL(rope_kernel, p), dim3(static_cast<unsigned>(grid)), dim3(kRopeThreads), 0, s, p);
}

// Sines and cosines of two angles up to pi / 4 by their Taylor series to y^9 and y^10
// (off by y^11 / 11! and y^12 / 12!: 2^-29 and 2^-33, against FP32's 2^-24).
PURO_DEV void sincos2(uint64_t y, uint64_t &sn, uint64_t &cs) {
    auto c = [](float x) { return f32x2(x, x); };
    const uint64_t z = mul_f32x2(y, y);
    uint64_t s = c(1.0f / 362880.0f), k = c(-1.0f / 3628800.0f);
    s = fma_f32x2(s, z, c(-1.0f / 5040.0f));
    k = fma_f32x2(k, z, c(1.0f / 40320.0f));
    s = fma_f32x2(s, z, c(1.0f / 120.0f));
    k = fma_f32x2(k, z, c(-1.0f / 720.0f));
    s = fma_f32x2(s, z, c(-1.0f / 6.0f));
    k = fma_f32x2(k, z, c(1.0f / 24.0f));
    k = fma_f32x2(k, z, c(-0.5f));
    sn = fma_f32x2(mul_f32x2(s, z), y, y);
    cs = fma_f32x2(k, z, c(1.0f));
}

// cos[i][j], sin[i][j] = scale times those of position first + i, four pairs of kRows
// positions a thread.  The fraction of a turn is taken from its nearest quarter in
// integers, so that the rest, up to an eighth of a turn, keeps 24 bits.  Bound by the
// writes: [131072, 64] in 10.4 us, 6.5 TB/s (with sincospif and a product for each pair 16.7).
constexpr int kTableThreads = 256, kTableRows = 4;
__global__ void __launch_bounds__(kTableThreads) rope_tables_kernel(const uint64_t *__restrict__ freq, int pairs, float scale, uint32_t first,
                                                                    int64_t count, float *__restrict__ cos, float *__restrict__ sin) {
    pdl_wait();
    pdl_launch_dependents();
    const int per = pairs / 4;  // threads a row
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kTableThreads + threadIdx.x;
    const int64_t row = i / per * kTableRows;
    if (row >= count) return;
    const int j = static_cast<int>(i % per) * 4;
    uint64_t f[4], turn[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f[k] = __ldg(freq + j + k);
        turn[k] = static_cast<uint64_t>(first + static_cast<uint32_t>(row)) * f[k];
    }
#pragma unroll
    for (int r = 0; r < kTableRows; ++r) {
        if (row + r >= count) break;
        float c[4], s[4];
        uint32_t quarter[4];
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t t = static_cast<uint32_t>(turn[k] >> 32);
            quarter[k] = (t + (1u << 29)) >> 30;
            y[k] = static_cast<float>(static_cast<int32_t>(t - (quarter[k] << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
            turn[k] += f[k];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint64_t sn, cs;
            sincos2(f32x2(y[2 * h], y[2 * h + 1]), sn, cs);
            split_f32x2(sn, s[2 * h], s[2 * h + 1]);
            split_f32x2(cs, c[2 * h], c[2 * h + 1]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool odd = quarter[k] & 1u;
            const float a = odd ? s[k] : c[k], b = odd ? c[k] : s[k];
            // the signs in the quarters 0 .. 3: cosine + - - +, sine + + - -
            c[k] = scale * __uint_as_float(__float_as_uint(a) ^ ((quarter[k] + 1u) << 30 & 0x80000000u));
            s[k] = scale * __uint_as_float(__float_as_uint(b) ^ (quarter[k] << 30 & 0x80000000u));
        }
        const int64_t at = (row + r) * pairs + j;
        *reinterpret_cast<float4 *>(cos + at) = make_float4(c[0], c[1], c[2], c[3]);
        *reinterpret_cast<float4 *>(sin + at) = make_float4(s[0], s[1], s[2], s[3]);
    }
}

cudaError_t launch_rope_tables(const uint64_t *freq, int pairs, float scale, int64_t first, int64_t count, float *cos, float *sin,
                               cudaStream_t s) {
    const int64_t grid = ((count + kTableRows - 1) / kTableRows * (pairs / 4) + kTableThreads - 1) / kTableThreads;
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_pdl(rope_tables_kernel, dim3(static_cast<unsigned>(grid)), dim3(kTableThreads), 0, s, freq, pairs, scale,
                      static_cast<uint32_t>(first), count, cos, sin);
}

}  // namespace puro
