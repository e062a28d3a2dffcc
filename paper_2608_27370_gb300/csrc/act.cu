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
constexpr int64_t kActBlocks = 152 * 4;      // blocks to aim for

ActBackwardPlan plan_act_backward(int64_t rows, int64_t cols) {
    const int64_t strips = (cols + kActCols - 1) / kActCols;
    int64_t slabs = std::max<int64_t>(1, std::min((rows + 31) / 32, (kActBlocks + strips - 1) / strips));
    const int64_t slab_rows = ((rows + slabs - 1) / slabs + kActRows - 1) / kActRows * kActRows;
    slabs = (rows + slab_rows - 1) / slab_rows;
    return ActBackwardPlan{static_cast<int>(slabs), slab_rows};
}

template <int ACT>
__global__ void __launch_bounds__(256) act_backward_kernel(const uint16_t *dy, const uint16_t *__restrict__ z,
                                                           int64_t rows, int64_t cols, int64_t slab_rows, uint16_t *dz,
                                                           float *__restrict__ partial) {
    pdl_wait();
    pdl_launch_dependents();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kActCols + 8 * tx;
    const int64_t r1 = min(rows, (static_cast<int64_t>(blockIdx.y) + 1) * slab_rows);
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (c < cols) {
#pragma unroll 4
        for (int64_t r = blockIdx.y * slab_rows + ty; r < r1; r += kActRows) {
            const int64_t at = r * cols + c;
            const uint4 d = __ldcg(reinterpret_cast<const uint4 *>(dy + at));  // (dz may be dy: past L1)
            uint4 zw = d;
            if constexpr (ACT != PURO_ACT_NONE) zw = __ldg(reinterpret_cast<const uint4 *>(z + at));
            uint4 o;
            o.x = act_backward2<ACT>(d.x, zw.x, sum[0], sum[1]);
            o.y = act_backward2<ACT>(d.y, zw.y, sum[2], sum[3]);
            o.z = act_backward2<ACT>(d.z, zw.z, sum[4], sum[5]);
            o.w = act_backward2<ACT>(d.w, zw.w, sum[6], sum[7]);
            if (dz) *reinterpret_cast<uint4 *>(dz + at) = ACT == PURO_ACT_NONE ? d : o;
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
    if (c < cols)
        for (int64_t k = ty; k < n; k += 8) a += partial[k * cols + c];
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

// [dgate, dup] of eight columns of one row a thread and step.
template <int ACT>
__global__ void __launch_bounds__(256) gated_backward_kernel(const uint16_t *__restrict__ dh, const uint16_t *__restrict__ gate,
                                                             const uint16_t *__restrict__ up, int64_t rows, int64_t cols,
                                                             int64_t ld, uint16_t *__restrict__ dgate_up) {
    pdl_wait();
    pdl_launch_dependents();
    const int64_t per_row = cols / 8, chunks = rows * per_row, stride = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < chunks; i += stride) {
        const int64_t r = i / per_row, c = (i - r * per_row) * 8;
        const uint4 d = __ldg(reinterpret_cast<const uint4 *>(dh) + i);
        const uint4 g = __ldg(reinterpret_cast<const uint4 *>(gate + r * ld + c)), u = __ldg(reinterpret_cast<const uint4 *>(up + r * ld + c));
        uint4 dg, du;
        dg.x = gate_backward2<ACT>(d.x, g.x, u.x), du.x = up_backward2<ACT>(d.x, g.x);
        dg.y = gate_backward2<ACT>(d.y, g.y, u.y), du.y = up_backward2<ACT>(d.y, g.y);
        dg.z = gate_backward2<ACT>(d.z, g.z, u.z), du.z = up_backward2<ACT>(d.z, g.z);
        dg.w = gate_backward2<ACT>(d.w, g.w, u.w), du.w = up_backward2<ACT>(d.w, g.w);
        uint16_t *out = dgate_up + r * 2 * cols + c;
        *reinterpret_cast<uint4 *>(out) = dg;
        *reinterpret_cast<uint4 *>(out + cols) = du;
    }
}

cudaError_t launch_gated_backward(const uint16_t *dh, const uint16_t *gate, const uint16_t *up, int64_t rows, int64_t cols,
                                  int64_t ld, int act, uint16_t *dgate_up, cudaStream_t s) {
    auto kern = act == PURO_ACT_RELU        ? gated_backward_kernel<PURO_ACT_RELU>
                : act == PURO_ACT_SILU      ? gated_backward_kernel<PURO_ACT_SILU>
                : act == PURO_ACT_GELU      ? gated_backward_kernel<PURO_ACT_GELU>
                : act == PURO_ACT_GELU_TANH ? gated_backward_kernel<PURO_ACT_GELU_TANH>
                                            : gated_backward_kernel<PURO_ACT_NONE>;
    const int64_t want = (rows * (cols / 8) + 255) / 256, cap = 152 * 8;
    return launch_pdl(kern, dim3(static_cast<unsigned>(want < cap ? want : cap)), dim3(256), 0, s, dh, gate, up, rows, cols, ld,
                      dgate_up);
}

}  // namespace puro
