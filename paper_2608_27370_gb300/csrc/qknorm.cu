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

constexpr int kQkFwdThreads = 128, kQkThreads = 256;  // (the backward's)
constexpr int kQkFwdBatch = 4, kQkBwdBatch = 2;       // heads of a token a group loads at once
// At most: two an SM are resident, each leaves a partial sum of a gain's gradient (a constant: it fixes the sums' order).
constexpr int kQkBwdBlocks = 152 * 2;
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

// The lane's sixteen channels as eight pairs (a, b), two pairs to a packed value:
// a[j] holds the first channels of pairs 2j and 2j + 1, b[j] the second.
struct Pairs {
    uint64_t a[4], b[4];
};
template <bool INTER>
PURO_DEV Pairs unpack16(const uint4 &w0, const uint4 &w1) {
    const uint32_t x[4] = {w0.x, w0.y, w0.z, w0.w}, y[4] = {w1.x, w1.y, w1.z, w1.w};
    Pairs p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (INTER) {  // neighbours: pairs 0 .. 3 in w0, 4 .. 7 in w1
            const uint32_t u = j < 2 ? x[2 * j] : y[2 * j - 4], v = j < 2 ? x[2 * j + 1] : y[2 * j - 3];
            p.a[j] = f32x2(bf16_lo(u), bf16_lo(v));
            p.b[j] = f32x2(bf16_hi(u), bf16_hi(v));
        } else {
            p.a[j] = f32x2(bf16_lo(x[j]), bf16_hi(x[j]));
            p.b[j] = f32x2(bf16_lo(y[j]), bf16_hi(y[j]));
        }
    }
    return p;
}

PURO_DEV uint32_t round2(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&b);
}
template <bool INTER>
PURO_DEV void pack16(const Pairs &p, uint4 &w0, uint4 &w1) {
    uint32_t x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a0, a1, b0, b1;
        split_f32x2(p.a[j], a0, a1);
        split_f32x2(p.b[j], b0, b1);
        if constexpr (INTER) {
            (j < 2 ? x : y)[2 * j & 3] = round2(a0, b0);
            (j < 2 ? x : y)[(2 * j & 3) + 1] = round2(a1, b1);
        } else {
            x[j] = round2(a0, a1);
            y[j] = round2(b0, b1);
        }
    }
    w0 = make_uint4(x[0], x[1], x[2], x[3]);
    w1 = make_uint4(y[0], y[1], y[2], y[3]);
}

// The angles of the lane's pairs: cosines, sines and negative sines.
struct Angles {
    uint64_t c[4], s[4], n[4];
};
// R p, or with s and n exchanged R^T p.
PURO_DEV void turn(Pairs &p, const uint64_t (&c)[4], const uint64_t (&s)[4], const uint64_t (&n)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint64_t a = p.a[j], b = p.b[j];
        p.a[j] = fma_f32x2(b, n[j], mul_f32x2(a, c[j]));
        p.b[j] = fma_f32x2(a, s[j], mul_f32x2(b, c[j]));
    }
}
PURO_DEV void scale(Pairs &p, uint64_t f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p.a[j] = mul_f32x2(p.a[j], f);
        p.b[j] = mul_f32x2(p.b[j], f);
    }
}
PURO_DEV void times(Pairs &p, const Pairs &q) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        p.a[j] = mul_f32x2(p.a[j], q.a[j]);
        p.b[j] = mul_f32x2(p.b[j], q.b[j]);
    }
}
// The sum of the products of the lane's channels.
PURO_DEV float dot(const Pairs &p, const Pairs &q) {
    uint64_t s = mul_f32x2(p.a[0], q.a[0]), t = mul_f32x2(p.b[0], q.b[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) {
        s = fma_f32x2(p.a[j], q.a[j], s);
        t = fma_f32x2(p.b[j], q.b[j], t);
    }
    float lo, hi;
    split_f32x2(add_f32x2(s, t), lo, hi);
    return lo + hi;
}

template <int G>
PURO_DEV float group_sum(float x) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// The token's position and angles.  A negative position marks a padding row
// (kRowPad); one past the tables cannot be rotated (kRowOut).
enum QkRow : int { kRowLive, kRowPad, kRowOut };
PURO_DEV QkRow qk_angles(const QkArgs &p, int64_t t, const QkLane &l, Angles &g) {
    const int64_t pos = p.positions ? __ldg(p.positions + t) : t;
    if (pos < 0) return kRowPad;
    if (p.rot > 0 && pos >= p.max_positions) return kRowOut;
    if (l.in && l.turned) {
        const float4 *c = reinterpret_cast<const float4 *>(p.cos + pos * (p.rot / 2) + l.pair);
        const float4 *s = reinterpret_cast<const float4 *>(p.sin + pos * (p.rot / 2) + l.pair);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float4 x = __ldg(c + k), y = __ldg(s + k);
            g.c[2 * k] = f32x2(x.x, x.y);
            g.c[2 * k + 1] = f32x2(x.z, x.w);
            g.s[2 * k] = f32x2(y.x, y.y);
            g.s[2 * k + 1] = f32x2(y.z, y.w);
            g.n[2 * k] = f32x2(-y.x, -y.y);
            g.n[2 * k + 1] = f32x2(-y.z, -y.w);
        }
    }
    return kRowLive;
}

// 1 / sqrt(x) (about 2^-23 off).
PURO_DEV float rsqrt_f32(float x) {
    float y;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a row that is not live counts as: zeros for padding, whatever it holds,
// and NaN past the tables.
PURO_DEV void replace_row(QkRow row, uint4 (&w)[2]) {
    const uint32_t v = row == kRowPad ? 0u : 0x7FC07FC0u;
    w[0] = w[1] = make_uint4(v, v, v, v);
}

// A block: some tokens' batch of heads of one kind, the batches of the same tokens
// next to one another (the queries' first).  On 8192 tokens of 16 + 8 heads of 128
// 20.6 us (5.0 TB/s), on 32768 of 12 + 2 heads 42.0 us (5.7 TB/s); the same loads and
// stores without the arithmetic take 16.4 and 35.3.  Blocks of 256 threads, three
// an SM: 22.1 and 44.7; batches of two, three, five, six heads 22.7, 21.6, 20.4, 20.8 (and
// more for one token, 2.3 us, or 1024).  Persistent blocks with the next items' loads
// in flight (cp.async, two ahead) took 23 to 45 us: what that saves goes into
// addresses.
template <int G, bool INTER>
__global__ void __launch_bounds__(kQkFwdThreads, 5) qk_norm_rope_kernel(const QkArgs p) {
    constexpr int B = kQkFwdBatch;
    pdl_wait();
    pdl_launch_dependents();
    const QkLane l = qk_lane(threadIdx.x % G, p.D, p.rot, INTER);
    const unsigned q_batches = (p.q.heads + B - 1) / B, batches = q_batches + (p.k.heads + B - 1) / B;
    const int64_t t = static_cast<int64_t>(blockIdx.x / batches) * (kQkFwdThreads / G) + threadIdx.x / G;
    const unsigned batch = blockIdx.x % batches;
    const bool is_q = batch < q_batches, live = t < p.tokens && l.in;
    const QkHeads &src = is_q ? p.q : p.k, &dst = is_q ? p.q_out : p.k_out;
    const int h0 = static_cast<int>(is_q ? batch : batch - q_batches) * B, n = min(B, src.heads - h0);
    const uint16_t *from = src.data + t * src.token_stride + h0 * src.head_stride;
    uint4 x[B][2];  // (y may be x: loaded past L1, where a neighbour's part of a sector would stay as it was)
#pragma unroll
    for (int b = 0; b < B; ++b) {
        x[b][0] = x[b][1] = make_uint4(0, 0, 0, 0);
        if (live && b < n) {
            x[b][0] = __ldcg(reinterpret_cast<const uint4 *>(from + l.o0));
            x[b][1] = __ldcg(reinterpret_cast<const uint4 *>(from + l.o1));
        }
        from += src.head_stride;
    }
    Angles ang;
    const QkRow row = live ? qk_angles(p, t, l, ang) : kRowPad;
    if (row != kRowLive) {
#pragma unroll
        for (int b = 0; b < B; ++b) replace_row(row, x[b]);
        if (row == kRowOut && p.status && l.pair == 0) *p.status = kQkStatusInvalid;
    }
    const float inv = 1.0f / static_cast<float>(p.D);
    const uint16_t *gains = is_q ? p.q_gain : p.k_gain;
    Pairs gain;
    if (gains && l.in)
        gain = unpack16<INTER>(__ldg(reinterpret_cast<const uint4 *>(gains + l.o0)), __ldg(reinterpret_cast<const uint4 *>(gains + l.o1)));
    uint16_t *to = dst.data + t * dst.token_stride + h0 * dst.head_stride;
    float *rstds = p.rstd + t * (p.q.heads + p.k.heads) + (is_q ? 0 : p.q.heads) + h0;
    const bool store_rstd = live && p.rstd && l.pair == 0, turned = row == kRowLive && l.turned;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        if (b >= n) break;  // the same for the whole block
        Pairs v = unpack16<INTER>(x[b][0], x[b][1]);
        float rstd = rsqrt_f32(fmaf(group_sum<G>(dot(v, v)), inv, p.eps));
        if (row == kRowPad) rstd = 0.0f;
        if (store_rstd) rstds[b] = rstd;
        if (gains) times(v, gain);
        scale(v, f32x2(rstd, rstd));
        if (turned) turn(v, ang.c, ang.s, ang.n);
        uint4 y0, y1;
        pack16<INTER>(v, y0, y1);
        if (live) {
            *reinterpret_cast<uint4 *>(to + l.o0) = y0;
            *reinterpret_cast<uint4 *>(to + l.o1) = y1;
        }
        to += dst.head_stride;
    }
}

// Blocks [0, p.q_blocks) take the query heads, the others the key heads, each a
// strided share of (token, batch of heads); so a thread sums one gain's
// gradient, in a fixed order, and a block leaves one partial sum [D].  8192 tokens
// of 16 + 8 heads of 128 30.8 us with the gains' sum (5.0 TB/s), 32768 of 12 + 2 heads
// 65.8 (5.4 TB/s); one, three, four heads a batch 37, 33, 33 us on the first.
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
    const int batches = (X.heads + B - 1) / B;
    const uint16_t *gain = is_q ? p.q_gain : p.k_gain;
    Pairs g = {};
    if (gain && l.in)
        g = unpack16<INTER>(__ldg(reinterpret_cast<const uint4 *>(gain + l.o0)), __ldg(reinterpret_cast<const uint4 *>(gain + l.o1)));
    const float inv = 1.0f / static_cast<float>(p.D);
    Pairs acc = {};  // (zero bits)
    // item = token * batches + batch; the next one is a step on, taken without a division
    const int64_t items = p.tokens * batches;
    const int step = blocks * kGroups, dt = step / batches, db = step - dt * batches;
    const int item0 = block * kGroups + threadIdx.x / G;
    int64_t t = item0 / batches;
    int batch = static_cast<int>(item0 - t * batches);
    for (int64_t i0 = static_cast<int64_t>(block) * kGroups; i0 < items; i0 += step) {
        const int h0 = batch * B;
        const bool live = t < p.tokens && l.in;
        uint4 x[B][2], dy[B][2];
        float rs[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            x[b][0] = x[b][1] = dy[b][0] = dy[b][1] = make_uint4(0, 0, 0, 0);
            rs[b] = 0.0f;
            if (live && h0 + b < X.heads) {
                const uint16_t *px = X.data + t * X.token_stride + (h0 + b) * X.head_stride;
                const uint16_t *py = DY.data + t * DY.token_stride + (h0 + b) * DY.head_stride;
                x[b][0] = *reinterpret_cast<const uint4 *>(px + l.o0);
                x[b][1] = *reinterpret_cast<const uint4 *>(px + l.o1);
                dy[b][0] = __ldcg(reinterpret_cast<const uint4 *>(py + l.o0));  // (dx may be dy: as above)
                dy[b][1] = __ldcg(reinterpret_cast<const uint4 *>(py + l.o1));
                rs[b] = __ldg(p.rstd + t * heads + first + h0 + b);
            }
        }
        Angles ang;
        const QkRow row = live ? qk_angles(p, t, l, ang) : kRowPad;
        if (row != kRowLive) {
#pragma unroll
            for (int b = 0; b < B; ++b) {
                replace_row(row, x[b]);
                replace_row(row, dy[b]);
                if (row == kRowPad) rs[b] = 0.0f;
            }
            if (row == kRowOut && p.status && l.pair == 0) *p.status = kQkStatusInvalid;
        }
        const bool turned = row == kRowLive && l.turned;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            Pairs d = unpack16<INTER>(dy[b][0], dy[b][1]), xh = unpack16<INTER>(x[b][0], x[b][1]);
            if (turned) turn(d, ang.c, ang.n, ang.s);
            scale(xh, f32x2(rs[b], rs[b]));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc.a[j] = fma_f32x2(d.a[j], xh.a[j], acc.a[j]);
                acc.b[j] = fma_f32x2(d.b[j], xh.b[j], acc.b[j]);
            }
            if (gain) times(d, g);
            const float m = -inv * group_sum<G>(dot(d, xh));
            const uint64_t mm = f32x2(m, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                d.a[j] = fma_f32x2(xh.a[j], mm, d.a[j]);
                d.b[j] = fma_f32x2(xh.b[j], mm, d.b[j]);
            }
            scale(d, f32x2(rs[b], rs[b]));
            uint4 y0, y1;
            pack16<INTER>(d, y0, y1);
            if (live && h0 + b < X.heads) {
                uint16_t *w = DX.data + t * DX.token_stride + (h0 + b) * DX.head_stride;
                *reinterpret_cast<uint4 *>(w + l.o0) = y0;
                *reinterpret_cast<uint4 *>(w + l.o1) = y1;
            }
        }
        t += dt;
        batch += db;
        if (batch >= batches) {
            batch -= batches;
            ++t;
        }
    }
    if (!p.partial) return;
    // the block's partial sum: over the groups of a warp, then over the warps in order
    __shared__ float part[kQkThreads / 32][16 * G];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v[4];  // first and second channels of pairs 2j and 2j + 1
        split_f32x2(acc.a[j], v[0], v[1]);
        split_f32x2(acc.b[j], v[2], v[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int o = G; o < 32; o <<= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
        }
        if ((threadIdx.x & 31) < G && l.in) {
            float *to = part[threadIdx.x / 32];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int pr = 2 * j + k;  // the lane's pair
                to[INTER ? l.o0 + 2 * pr : l.o0 + pr] = v[k];
                to[INTER ? l.o0 + 2 * pr + 1 : l.o1 + pr] = v[2 + k];
            }
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += kQkThreads) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kQkThreads / 32; ++w) s += part[w][c];
        p.partial[static_cast<int64_t>(blockIdx.x) * p.D + c] = s;
    }
}

// dgain = the blocks' partial sums: 32 columns a block, 32 interleaved shares of
// the partial sums each, then the shares in order.
__global__ void __launch_bounds__(1024) qk_gain_kernel(const float *__restrict__ partial, int D, int q_blocks, int blocks,
                                                       float *__restrict__ dq_gain, float *__restrict__ dk_gain) {
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float part[32][33];
    const int from = blockIdx.y ? q_blocks : 0, n = blockIdx.y ? blocks - q_blocks : q_blocks;
    float *out = blockIdx.y ? dk_gain : dq_gain;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = 32 * blockIdx.x + tx;
    constexpr int kMost = (kQkBwdBlocks + 31) / 32;
    float v[kMost];  // (all of a share's loads at once: one latency)
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int b = ty + 32 * i;
        v[i] = c < D && b < n ? partial[static_cast<int64_t>(from + b) * D + c] : 0.0f;
    }
    float a = v[0];
#pragma unroll
    for (int i = 1; i < kMost; ++i) a += v[i];
    part[ty][tx] = a;
    __syncthreads();
    if (ty != 0 || c >= D || !out) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) a += part[k][tx];
    out[c] = a;
}

static int group_lanes(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// Blocks for the query and key heads of the backward pass; host-only, by shape
// alone (the partial sums' order is fixed by it).
void qk_backward_blocks(int64_t tokens, int q_heads, int k_heads, int D, int *q_blocks, int *blocks) {
    const int64_t groups = kQkThreads / group_lanes(D), most = kQkBwdBlocks;
    auto need = [&](int heads) { return (tokens * ((heads + kQkBwdBatch - 1) / kQkBwdBatch) + groups - 1) / groups; };
    const int64_t nq = need(q_heads), nk = need(k_heads);
    if (nq + nk <= most) {
        *q_blocks = static_cast<int>(nq);
        *blocks = static_cast<int>(nq + nk);
        return;
    }
    const int64_t q = (most * nq + (nq + nk) / 2) / (nq + nk);
    *q_blocks = static_cast<int>(nk == 0 ? most : nq == 0 ? 0 : std::max<int64_t>(1, std::min<int64_t>(most - 1, q)));
    *blocks = static_cast<int>(most);
}

// kern<G, INTER> for the group's lanes and the kind of pairs
#define PURO_QK_KERNEL(kern, p)                                                                      \
    (group_lanes((p).D) == 4   ? ((p).inter ? kern<4, true> : kern<4, false>)                         \
     : group_lanes((p).D) == 8 ? ((p).inter ? kern<8, true> : kern<8, false>)                         \
                               : ((p).inter ? kern<16, true> : kern<16, false>))

cudaError_t launch_qk_norm_rope(const QkArgs &p, cudaStream_t s) {
    const int64_t per = kQkFwdThreads / group_lanes(p.D);
    auto batches = [](int heads) { return (heads + kQkFwdBatch - 1) / kQkFwdBatch; };
    const int64_t grid = (p.tokens + per - 1) / per * (batches(p.q.heads) + batches(p.k.heads));
    if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_pdl(PURO_QK_KERNEL(qk_norm_rope_kernel, p), dim3(static_cast<unsigned>(grid)), dim3(kQkFwdThreads), 0, s, p);
}

cudaError_t launch_qk_norm_rope_backward(QkArgs p, float *dq_gain, float *dk_gain, cudaStream_t s) {
    int blocks = 0;
    qk_backward_blocks(p.tokens, p.q.heads, p.k.heads, p.D, &p.q_blocks, &blocks);
    if (blocks > 0) {
        const cudaError_t e =
            launch_pdl(PURO_QK_KERNEL(qk_norm_rope_backward_kernel, p), dim3(blocks), dim3(kQkThreads), 0, s, p);
        if (e != cudaSuccess) return e;
    }
    if (!(dq_gain || dk_gain)) return cudaSuccess;
    return launch_pdl(qk_gain_kernel, dim3((p.D + 31) / 32, 2), dim3(1024), 0, s, static_cast<const float *>(p.partial), p.D,
                      p.q_blocks, blocks, dq_gain, dk_gain);
}

}  // namespace puro
