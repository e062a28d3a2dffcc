// qknorm.cu -- RMSNorm of each query and key head with the position rotation
// in the same pass, and its backward (Puro-2B, section "Model architecture and
// pretraining system": the Qwen3 architecture normalises queries and keys head
// by head before it rotates them).
//
// Per token t and head, D channels:
//   rstd = 1 / sqrt(mean(x^2) + eps),  n = (x * rstd) * gain,  y = R(pos_t) n
// R turns the pairs (i, i + rot/2) of the first rot channels (or the neighbours
// (2i, 2i + 1)) by the position's angles, cos and sin from tables; the other
// channels pass.  Backward, with xh = x * rstd:
//   dn = R^T dy,  dgain = sum over tokens and heads of dn * xh,
//   dx = rstd * (dn * gain - xh * mean(dn * gain * xh)).
// All of it is in FP32; y and dx are rounded to BF16 once.
//
// Bound by memory: x is read once and y written once (backward: x and dy read,
// dx written).  A head belongs to a group of G lanes, 16 channels a lane in two
// 16-byte chunks that hold both channels of each of its pairs, so the rotation
// needs no exchange between lanes and the norm one butterfly over the group.  A
// group takes the heads of one token in batches whose loads are all issued
// first; the token's angles stay in registers for the batch.
#include <cuda_bf16.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "quant_math.cuh"

namespace puro {

constexpr int kQkThreads = 256;
constexpr int kQkFwdBatch = 4;   // heads of a token a group loads at once
constexpr int kQkBwdBatch = 2;
constexpr int kQkBwdBlocks = 152 * 2;  // at most: two an SM are resident, each leaves a partial sum of a gain's gradient
constexpr int32_t kQkStatusInvalid = 1;  // PURO_ERR_INVALID_ARG

// The lane's channels: two chunks of eight, at o0 and o1 of the head, and the
// first of the eight pairs (so of the table's columns) they make up.
struct QkLane {
    int o0, o1, pair;
    bool in, turned;
};
PURO_DEV QkLane qk_lane(int c, int D, int rot, int inter) {
    QkLane l;
    l.in = 16 * c < D;
    l.turned = 16 * c < rot;
    l.pair = 8 * c;
    l.o0 = l.turned && !inter ? 8 * c : 16 * c;
    l.o1 = l.turned && !inter ? rot / 2 + 8 * c : 16 * c + 8;
    return l;
}

PURO_DEV void load8(const float *p, float (&v)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

PURO_DEV void widen8(const uint4 &w, float *v) {
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(ws[i]);
        v[2 * i + 1] = bf16_hi(ws[i]);
    }
}

PURO_DEV uint4 narrow8(const float *v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// R v (sign 1) or R^T v (sign -1) of the lane's sixteen channels.
PURO_DEV void turn16(float (&v)[16], const float (&co)[8], const float (&si)[8], bool inter, float sign) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = sign * si[i];
        const float a = inter ? v[2 * i] : v[i], b = inter ? v[2 * i + 1] : v[8 + i];
        const float p = a * co[i] - b * s, q = b * co[i] + a * s;
        if (inter) {
            v[2 * i] = p;
            v[2 * i + 1] = q;
        } else {
            v[i] = p;
            v[8 + i] = q;
        }
    }
}

template <int G>
PURO_DEV float group_sum(float x) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// The token's position and angles.  A negative position marks a padding row
// (kPad); one past the tables cannot be rotated (kOut).
enum QkRow : int { kRowLive, kRowPad, kRowOut };
PURO_DEV QkRow qk_angles(const QkArgs &p, int64_t t, const QkLane &l, float (&co)[8], float (&si)[8]) {
    const int64_t pos = p.positions ? __ldg(p.positions + t) : t;
    if (pos < 0) return kRowPad;
    if (p.rot > 0 && pos >= p.max_positions) return kRowOut;
    if (l.in && l.turned) {
        load8(p.cos + pos * (p.rot / 2) + l.pair, co);
        load8(p.sin + pos * (p.rot / 2) + l.pair, si);
    }
    return kRowLive;
}

PURO_DEV float nan_f32() { return __uint_as_float(0x7FC00000u); }

template <int G, bool INTER>
__global__ void __launch_bounds__(kQkThreads) qk_norm_rope_kernel(const QkArgs p) {
    constexpr int B = kQkFwdBatch;
    pdl_wait();
    pdl_launch_dependents();
    const QkLane l = qk_lane(threadIdx.x % G, p.D, p.rot, INTER);
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (kQkThreads / G) + threadIdx.x / G;
    const int h0 = blockIdx.y * B, heads = p.q.heads + p.k.heads;
    const bool live = t < p.tokens;
    uint4 x[B][2];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int h = h0 + b;
        x[b][0] = x[b][1] = make_uint4(0, 0, 0, 0);
        if (live && l.in && h < heads) {
            const QkHeads &src = h < p.q.heads ? p.q : p.k;
            const uint16_t *r = src.data + t * src.token_stride + (h < p.q.heads ? h : h - p.q.heads) * src.head_stride;
            x[b][0] = *reinterpret_cast<const uint4 *>(r + l.o0);
            x[b][1] = *reinterpret_cast<const uint4 *>(r + l.o1);
        }
    }
    float co[8], si[8];
    const QkRow row = live ? qk_angles(p, t, l, co, si) : kRowPad;
    if (row == kRowOut && p.status && l.pair == 0) *p.status = kQkStatusInvalid;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int h = h0 + b;
        if (h >= heads) break;  // the same for the whole block
        float v[16];
        widen8(x[b][0], v);
        widen8(x[b][1], v + 8);
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s0 = fmaf(v[i], v[i], s0);
            s1 = fmaf(v[8 + i], v[8 + i], s1);
        }
        const float ss = group_sum<G>(s0 + s1);
        float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(ss, static_cast<float>(p.D)) + p.eps));
        if (row == kRowPad) rstd = 0.0f;
        if (row == kRowOut) rstd = nan_f32();
        const bool is_q = h < p.q.heads;
        if (live && p.rstd && l.pair == 0) p.rstd[t * heads + h] = rstd;
        if (!live || !l.in) continue;
        const uint16_t *gain = is_q ? p.q_gain : p.k_gain;
        if (gain) {
            float g[16];
            widen8(__ldg(reinterpret_cast<const uint4 *>(gain + l.o0)), g);
            widen8(__ldg(reinterpret_cast<const uint4 *>(gain + l.o1)), g + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = v[i] * rstd * g[i];
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= rstd;
        }
        if (row == kRowLive && l.turned) turn16(v, co, si, INTER, 1.0f);
        uint4 y0 = narrow8(v), y1 = narrow8(v + 8);
        if (row == kRowPad) y0 = y1 = make_uint4(0, 0, 0, 0);  // whatever the row holds
        const QkHeads &dst = is_q ? p.q_out : p.k_out;
        uint16_t *w = dst.data + t * dst.token_stride + (is_q ? h : h - p.q.heads) * dst.head_stride;
        *reinterpret_cast<uint4 *>(w + l.o0) = y0;
        *reinterpret_cast<uint4 *>(w + l.o1) = y1;
    }
}

// Blocks [0, p.q_blocks) take the query heads, the others the key heads, each a
// strided share of (token, batch of heads); so a thread sums one gain's
// gradient, in a fixed order, and a block leaves one partial sum [D].
template <int G, bool INTER>
__global__ void __launch_bounds__(kQkThreads, 2) qk_norm_rope_backward_kernel(const QkArgs p) {
    constexpr int B = kQkBwdBatch, kGroups = kQkThreads / G;
    pdl_wait();
    pdl_launch_dependents();
    const QkLane l = qk_lane(threadIdx.x % G, p.D, p.rot, INTER);
    const bool is_q = static_cast<int>(blockIdx.x) < p.q_blocks;
    const int block = is_q ? blockIdx.x : blockIdx.x - p.q_blocks;
    const int blocks = is_q ? p.q_blocks : gridDim.x - p.q_blocks;
    const QkHeads &X = is_q ? p.q : p.k, &DY = is_q ? p.q_out : p.k_out, &DX = is_q ? p.dq : p.dk;
    const int first = is_q ? 0 : p.q.heads, heads = p.q.heads + p.k.heads;
    const int64_t batches = (X.heads + B - 1) / B;
    const uint16_t *gain = is_q ? p.q_gain : p.k_gain;
    uint4 gw[2] = {};
    if (gain && l.in) {
        gw[0] = __ldg(reinterpret_cast<const uint4 *>(gain + l.o0));
        gw[1] = __ldg(reinterpret_cast<const uint4 *>(gain + l.o1));
    }
    float acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    const int64_t items = p.tokens * batches, step = static_cast<int64_t>(blocks) * kGroups;
    for (int64_t i0 = static_cast<int64_t>(block) * kGroups; i0 < items; i0 += step) {
        const int64_t item = i0 + threadIdx.x / G;
        const int64_t t = item / batches;
        const int h0 = static_cast<int>(item - t * batches) * B;
        const bool live = item < items;
        uint4 x[B][2], dy[B][2];
        float rs[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            x[b][0] = x[b][1] = dy[b][0] = dy[b][1] = make_uint4(0, 0, 0, 0);
            rs[b] = 0.0f;
            if (live && l.in && h0 + b < X.heads) {
                const uint16_t *px = X.data + t * X.token_stride + (h0 + b) * X.head_stride;
                const uint16_t *py = DY.data + t * DY.token_stride + (h0 + b) * DY.head_stride;
                x[b][0] = *reinterpret_cast<const uint4 *>(px + l.o0);
                x[b][1] = *reinterpret_cast<const uint4 *>(px + l.o1);
                dy[b][0] = *reinterpret_cast<const uint4 *>(py + l.o0);
                dy[b][1] = *reinterpret_cast<const uint4 *>(py + l.o1);
                rs[b] = __ldg(p.rstd + t * heads + first + h0 + b);
            }
        }
        float co[8], si[8];
        const QkRow row = live ? qk_angles(p, t, l, co, si) : kRowPad;
        if (row == kRowOut && p.status && l.pair == 0) *p.status = kQkStatusInvalid;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            float d[16], xh[16], g[16];
            widen8(dy[b][0], d);
            widen8(dy[b][1], d + 8);
            widen8(x[b][0], xh);
            widen8(x[b][1], xh + 8);
            widen8(gw[0], g);
            widen8(gw[1], g + 8);
            if (row == kRowLive && l.turned) turn16(d, co, si, INTER, -1.0f);
            const float r = row == kRowOut ? nan_f32() : rs[b];
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                xh[i] *= r;
                if (row != kRowPad) acc[i] = fmaf(d[i], xh[i], acc[i]);
                if (gain) d[i] *= g[i];
                if (i < 8)
                    s0 = fmaf(d[i], xh[i], s0);
                else
                    s1 = fmaf(d[i], xh[i], s1);
            }
            const float m = group_sum<G>(s0 + s1) / static_cast<float>(p.D);
            if (!live || !l.in || h0 + b >= X.heads) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = r * (d[i] - xh[i] * m);
            uint4 y0 = narrow8(d), y1 = narrow8(d + 8);
            if (row == kRowPad) y0 = y1 = make_uint4(0, 0, 0, 0);
            uint16_t *w = DX.data + t * DX.token_stride + (h0 + b) * DX.head_stride;
            *reinterpret_cast<uint4 *>(w + l.o0) = y0;
            *reinterpret_cast<uint4 *>(w + l.o1) = y1;
        }
    }
    if (!p.partial) return;
    // the block's partial sum: over the groups of a warp, then over the warps in order
    __shared__ float part[kQkThreads / 32][16 * G];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int o = G; o < 32; o <<= 1) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
    }
    if ((threadIdx.x & 31) < G && l.in) {
#pragma unroll
        for (int i = 0; i < 16; ++i) part[threadIdx.x / 32][(i < 8 ? l.o0 : l.o1 - 8) + i] = acc[i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += kQkThreads) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kQkThreads / 32; ++w) s += part[w][c];
        p.partial[static_cast<int64_t>(blockIdx.x) * p.D + c] = s;
    }
}

// dgain = the blocks' partial sums, eight slices of them in block order and the
// slices in order.  One block each for the queries' and the keys' gain.
__global__ void __launch_bounds__(1024) qk_gain_kernel(const float *__restrict__ partial, int D, int q_blocks, int blocks,
                                                       float *__restrict__ dq_gain, float *__restrict__ dk_gain) {
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float part[1024];
    const int from = blockIdx.x ? q_blocks : 0, n = blockIdx.x ? blocks - q_blocks : q_blocks;
    float *out = blockIdx.x ? dk_gain : dq_gain;
    const int slices = 1024 / D;
    const int c = threadIdx.x % D, s = threadIdx.x / D;
    float a = 0.0f;
    if (s < slices)
        for (int b = s; b < n; b += slices) a += partial[static_cast<int64_t>(from + b) * D + c];
    part[threadIdx.x] = a;
    __syncthreads();
    if (s == 0 && out) {
        for (int k = 1; k < slices; ++k) a += part[k * D + c];
        out[c] = a;
    }
}

static int group_lanes(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// Blocks for the query and key heads of the backward pass; host-only, by shape
// alone (the partial sums' order is fixed by it).
void qk_backward_blocks(int64_t tokens, int q_heads, int k_heads, int D, int *q_blocks, int *blocks) {
    const int64_t groups = kQkThreads / group_lanes(D);
    auto need = [&](int heads) { return (tokens * ((heads + kQkBwdBatch - 1) / kQkBwdBatch) + groups - 1) / groups; };
    const int64_t nq = need(q_heads), nk = need(k_heads);
    if (nq + nk <= kQkBwdBlocks) {
        *q_blocks = static_cast<int>(nq);
        *blocks = static_cast<int>(nq + nk);
        return;
    }
    int64_t q = k_heads == 0 ? kQkBwdBlocks : q_heads == 0 ? 0 : std::max<int64_t>(1, std::min<int64_t>(kQkBwdBlocks - 1, (kQkBwdBlocks * nq + (nq + nk) / 2) / (nq + nk)));
    *q_blocks = static_cast<int>(q);
    *blocks = kQkBwdBlocks;
}

template <int G>
static cudaError_t launch_fwd(const QkArgs &p, cudaStream_t s) {
    const int64_t per = kQkThreads / G;
    const dim3 grid(static_cast<unsigned>((p.tokens + per - 1) / per), (p.q.heads + p.k.heads + kQkFwdBatch - 1) / kQkFwdBatch);
    return launch_pdl(p.inter ? qk_norm_rope_kernel<G, true> : qk_norm_rope_kernel<G, false>, grid, dim3(kQkThreads), 0, s, p);
}

template <int G>
static cudaError_t launch_bwd(const QkArgs &p, int blocks, cudaStream_t s) {
    return launch_pdl(p.inter ? qk_norm_rope_backward_kernel<G, true> : qk_norm_rope_backward_kernel<G, false>, dim3(blocks),
                      dim3(kQkThreads), 0, s, p);
}

cudaError_t launch_qk_norm_rope(const QkArgs &p, cudaStream_t s) {
    switch (group_lanes(p.D)) {
        case 4: return launch_fwd<4>(p, s);
        case 8: return launch_fwd<8>(p, s);
        default: return launch_fwd<16>(p, s);
    }
}

cudaError_t launch_qk_norm_rope_backward(QkArgs p, float *dq_gain, float *dk_gain, cudaStream_t s) {
    int blocks = 0;
    qk_backward_blocks(p.tokens, p.q.heads, p.k.heads, p.D, &p.q_blocks, &blocks);
    cudaError_t e = cudaSuccess;
    if (blocks > 0) switch (group_lanes(p.D)) {
            case 4: e = launch_bwd<4>(p, blocks, s); break;
            case 8: e = launch_bwd<8>(p, blocks, s); break;
            default: e = launch_bwd<16>(p, blocks, s);
        }
    if (e != cudaSuccess || !(dq_gain || dk_gain)) return e;
    return launch_pdl(qk_gain_kernel, dim3(2), dim3(1024), 0, s, static_cast<const float *>(p.partial), p.D, p.q_blocks, blocks,
                      dq_gain, dk_gain);
}

}  // namespace puro
