// act.cu -- backward of a linear's bias and activation, and of the gate of the
// gated MLP (Puro-2B, section "Model architecture and pretraining system"), in
// BF16; quantize.cu has the forms that emit FP8 copies.
//   dz = dy * act'(z),                 dbias[c] = sum over rows of dz[:, c]
//   dgate = dh * up * act'(gate),      dup = dh * act(gate)
// Bound by memory: every input read once, every output written once; a thread
// takes eight columns (16 bytes) of a row.  The bias's gradient sums FP32
// values that are not rounded: a thread over the rows of its slab, a block over
// its eight rows of threads, then the slabs in order, so always in one order.
#include <cuda_bf16.h>

#include <algorithm>

#include "act_math.cuh"
#include "internal.h"
#include "ptx.cuh"

namespace puro {

constexpr int kActCols = 256;                // columns of a block: 32 threads of eight
constexpr int kActRows = 8;                  // rows of threads
constexpr int kActBatch = 2;                 // rows of a thread loaded at once
constexpr int64_t kActBlocks = 152 * 4;      // blocks at most: four an SM are resident (a constant: it fixes the sums' order)
constexpr int kGateBlocks = 4;               // of the gate's kernel an SM

ActBackwardPlan plan_act_backward(int64_t rows, int64_t cols) {
    const int64_t strips = (cols + kActCols - 1) / kActCols;
    int64_t slabs = std::max<int64_t>(1, std::min((rows + 31) / 32, kActBlocks / strips));
    const int64_t slab_rows = ((rows + slabs - 1) / slabs + kActRows - 1) / kActRows * kActRows;
    slabs = (rows + slab_rows - 1) / slab_rows;
    return ActBackwardPlan{static_cast<int>(slabs), slab_rows};
}

// Two rows of a thread at once, four blocks an SM.  With dbias, us at one / two / three /
// four rows: SiLU [8192, 8960] 72.1 / 70.9 / 69.7 / 80.6, none 57.6 / 48.8 / 51.2 / 50.8, GELU
// [1001, 1544] 6.4 / 6.1 / 7.2 / 7.0 (floors 65.0, 43.3, 1.4); five and six blocks no better;
// with a row's loads behind the stores of the one before 147, 56, 7.0.  (Of narrower sigmoids
// and a shorter GELU; two rows now 69.0, 49.2, 6.3.)
template <int ACT>
__global__ void __launch_bounds__(256, 4) act_backward_kernel(const uint16_t *dy, const uint16_t *__restrict__ z,
                                                           int64_t rows, int64_t cols, int64_t slab_rows, uint16_t *dz,
                                                           float *__restrict__ partial) {
    pdl_wait();
    pdl_launch_dependents();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kActCols + 8 * tx;
    const int64_t r1 = min(rows, (static_cast<int64_t>(blockIdx.y) + 1) * slab_rows);
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (c < cols) {
        for (int64_t r0 = blockIdx.y * slab_rows + ty; r0 < r1; r0 += kActBatch * kActRows) {
            uint4 d[kActBatch], zw[kActBatch];  // (all loads ahead of the stores, since dz may be dy; dy past L1 for the same reason)
#pragma unroll
            for (int b = 0; b < kActBatch; ++b) {
                const int64_t r = r0 + b * kActRows, at = r * cols + c;
                d[b] = r < r1 ? __ldcg(reinterpret_cast<const uint4 *>(dy + at)) : make_uint4(0u, 0u, 0u, 0u);
                zw[b] = ACT != PURO_ACT_NONE && r < r1 ? __ldg(reinterpret_cast<const uint4 *>(z + at)) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int b = 0; b < kActBatch; ++b) {
                const int64_t r = r0 + b * kActRows, at = r * cols + c;
                uint4 o;
                o.x = act_backward2<ACT>(d[b].x, zw[b].x, sum[0], sum[1]);
                o.y = act_backward2<ACT>(d[b].y, zw[b].y, sum[2], sum[3]);
                o.z = act_backward2<ACT>(d[b].z, zw[b].z, sum[4], sum[5]);
                o.w = act_backward2<ACT>(d[b].w, zw[b].w, sum[6], sum[7]);
                if (dz && r < r1) *reinterpret_cast<uint4 *>(dz + at) = ACT == PURO_ACT_NONE ? d[b] : o;
            }
        }
    }
    if (!partial) return;
    __shared__ float part[kActRows][kActCols];
#pragma unroll
    for (int i = 0; i < 8; ++i) part[ty][8 * tx + i] = sum[i];
    __syncthreads();
    const int64_t oc = static_cast<int64_t>(blockIdx.x) * kActCols + threadIdx.x;
    if (oc >= cols) return;
    float a = part[0][threadIdx.x];
#pragma unroll
    for (int k = 1; k < kActRows; ++k) a += part[k][threadIdx.x];
    partial[blockIdx.y * cols + oc] = a;
}

cudaError_t launch_act_backward(const uint16_t *dy, const uint16_t *z, int64_t rows, int64_t cols, int act, uint16_t *dz,
                                float *partial, cudaStream_t s) {
    const ActBackwardPlan plan = plan_act_backward(rows, cols);
    auto kern = act == PURO_ACT_RELU        ? act_backward_kernel<PURO_ACT_RELU>
                : act == PURO_ACT_SILU      ? act_backward_kernel<PURO_ACT_SILU>
                : act == PURO_ACT_GELU      ? act_backward_kernel<PURO_ACT_GELU>
                : act == PURO_ACT_GELU_TANH ? act_backward_kernel<PURO_ACT_GELU_TANH>
                                            : act_backward_kernel<PURO_ACT_NONE>;
    return launch_pdl(kern, dim3(static_cast<unsigned>((cols + kActCols - 1) / kActCols), plan.slabs), dim3(256), 0, s, dy, z,
                      rows, cols, plan.slab_rows, dz, partial);
}

// 32 columns a block, eight interleaved shares of the partial sums each.
__global__ void __launch_bounds__(256) column_sums_kernel(const float *__restrict__ partial, int64_t n, int64_t cols,
                                                          float *__restrict__ out) {
    pdl_wait();
    pdl_launch_dependents();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + tx;
    float a = 0.0f;
    for (int64_t k0 = ty; k0 < n; k0 += 64) {  // (eight loads at once: a latency for each 64 sums)
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c < cols && k0 + 8 * i < n ? partial[(k0 + 8 * i) * cols + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) a += v[i];
    }
    __shared__ float part[8][32];
    part[ty][tx] = a;
    __syncthreads();
    if (ty == 0 && c < cols) {
#pragma unroll
        for (int k = 1; k < 8; ++k) a += part[k][tx];
        out[c] = a;
    }
}

cudaError_t launch_column_sums(const float *partial, int64_t n, int64_t cols, float *dbias, cudaStream_t s) {
    return launch_pdl(column_sums_kernel, dim3(static_cast<unsigned>((cols + 31) / 32)), dim3(256), 0, s, partial, n, cols, dbias);
}

// [dgate, dup] of eight columns of a row a thread and step.  Blocks an SM, and us at
// four / five / six: SiLU [8192, 6144] 74.9 / 81.0 / 75.1, [777, 6144] 9.2 / 9.0 / 9.4, tanh
// GELU 74.7 / 78.9 / 80.2 and 9.2 / 10.1 / 10.2; GELU at four / six 77.0 / 81.2 and 9.6 / 9.8
// (floors 74.2 and 7.0; eight with a division a step and SiLU 91.6 and 10.6).  (Of narrower
// sigmoids and a shorter GELU; four now 75.0 and 9.2, 75.4 and 9.4, 79.1 and 10.0.)
template <int ACT>
__global__ void __launch_bounds__(256, kGateBlocks) gated_backward_kernel(const uint16_t *__restrict__ dh,
                                                                       const uint16_t *__restrict__ gate,
                                                                       const uint16_t *__restrict__ up, int64_t rows, int64_t cols,
                                                                       int64_t ld, uint16_t *__restrict__ dgate_up) {
    pdl_wait();
    pdl_launch_dependents();
    // chunk c (of eight columns) of row r; the next one is a step on, taken without a division
    const int64_t per_row = cols / 8, step = static_cast<int64_t>(gridDim.x) * blockDim.x, dr = step / per_row, dc = step - dr * per_row;
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    for (int64_t r = i0 / per_row, c = i0 - r * per_row; r < rows;) {
        const uint4 d = __ldg(reinterpret_cast<const uint4 *>(dh + r * cols + 8 * c));
        const uint4 g = __ldg(reinterpret_cast<const uint4 *>(gate + r * ld + 8 * c));
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(up + r * ld + 8 * c));
        uint4 dg, du;
        dg.x = gate_backward2<ACT>(d.x, g.x, u.x), du.x = up_backward2<ACT>(d.x, g.x);
        dg.y = gate_backward2<ACT>(d.y, g.y, u.y), du.y = up_backward2<ACT>(d.y, g.y);
        dg.z = gate_backward2<ACT>(d.z, g.z, u.z), du.z = up_backward2<ACT>(d.z, g.z);
        dg.w = gate_backward2<ACT>(d.w, g.w, u.w), du.w = up_backward2<ACT>(d.w, g.w);
        uint16_t *out = dgate_up + r * 2 * cols + 8 * c;
        *reinterpret_cast<uint4 *>(out) = dg;
        *reinterpret_cast<uint4 *>(out + cols) = du;
        r += dr, c += dc;
        if (c >= per_row) c -= per_row, ++r;
    }
}

cudaError_t launch_gated_backward(const uint16_t *dh, const uint16_t *gate, const uint16_t *up, int64_t rows, int64_t cols,
                                  int64_t ld, int act, uint16_t *dgate_up, cudaStream_t s) {
    auto kern = act == PURO_ACT_RELU        ? gated_backward_kernel<PURO_ACT_RELU>
                : act == PURO_ACT_SILU      ? gated_backward_kernel<PURO_ACT_SILU>
                : act == PURO_ACT_GELU      ? gated_backward_kernel<PURO_ACT_GELU>
                : act == PURO_ACT_GELU_TANH ? gated_backward_kernel<PURO_ACT_GELU_TANH>
                                            : gated_backward_kernel<PURO_ACT_NONE>;
    const int64_t want = (rows * (cols / 8) + 255) / 256, cap = static_cast<int64_t>(sm_count_here()) * kGateBlocks;
    return launch_pdl(kern, dim3(static_cast<unsigned>(want < cap ? want : cap)), dim3(256), 0, s, dh, gate, up, rows, cols, ld,
                      dgate_up);
}

}  // namespace puro
