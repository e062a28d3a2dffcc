// skinny.cu -- BF16 linears of a few tokens, with the epilogue (bias, activation,
// residual) or as the gated MLP's two projections: the form for single tokens.
//
// With a few tokens a linear is bound by reading its weight once: 2NK bytes at
// HBM's rate, far below the tensor cores'.  So no tile is staged: a warp streams
// eight rows of W (16 bytes a lane, four lanes a row) straight into the B
// fragments of mma.sync m16n8k16 and the tokens, which stay in L1, into the A
// fragments.  A product does not depend on the order of its terms, so a lane's
// eight consecutive k are taken as the k slots that its fragments hold (the same
// ones for A and B) and no shuffle is needed.  The reduction is split over the
// block's warps, whose partial sums meet in shared memory in warp order.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "act_math.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "quant_math.cuh"
#include "skinny_plan.h"

namespace puro {

// Weights are read once by one block: past L1, which the tokens keep.
PURO_DEV uint4 load_weights(const uint16_t *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// c += A B: A 16 x 16 (a: rows g and g + 8 of lane 4g + c), B 16 x 8.
PURO_DEV void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int skinny_unroll(bool gated) { return gated ? 2 : 3; }  // steps of 32 k that a warp loads at once

// One block: columns 8 blockIdx.x .. + 7 of the output (GATED: of h, from those
// rows of the gate and of up).  Up to 8 ROWS tokens.
template <int WARPS, bool GATED, int ROWS>
__global__ void __launch_bounds__(WARPS * 32) skinny_linear_kernel(const uint16_t *__restrict__ x, const uint16_t *__restrict__ w,
                                                                  int M, int N, int K, const GemmEpilogue epi) {
    constexpr int kTiles = GATED ? 2 : 1, kUnroll = skinny_unroll(GATED);
    constexpr int kMmas = (ROWS + 1) / 2;  // of sixteen tokens
    __shared__ float part[WARPS][kTiles][8 * ROWS][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int n0 = 8 * blockIdx.x;
    const uint16_t *wp[kTiles];
    wp[0] = w + static_cast<int64_t>(n0 + g) * K + 8 * c;
    if constexpr (GATED) wp[1] = wp[0] + static_cast<int64_t>(N) * K;
    const uint16_t *xp = x + static_cast<int64_t>(g) * K + 8 * c;
    const int steps = (K + 31) / 32, each = (steps + WARPS - 1) / WARPS;  // of 32 k, and a warp's share
    const int first = warp * each, last = min(steps, first + each);
    float acc[kTiles][kMmas][2][4] = {};
    // All of the warp's weights into L2 at once, ahead of the wait for the kernel
    // before (nothing is delivered, so they may still be being written): its loads
    // then find them there, whatever the registers hold in flight.
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
        for (int k = 32 * first + 64 * c; k < min(K, 32 * last); k += 256) prefetch_l2(wp[t] - 8 * c + k);
    pdl_wait();
    pdl_launch_dependents();
    for (int s0 = first; s0 < last; s0 += kUnroll) {
        uint4 b[kTiles][kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = 32 * (s0 + u);
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                b[t][u] = s0 + u < last && k + 8 * c < K ? load_weights(wp[t] + k) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = 32 * (s0 + u);
            const bool in = s0 + u < last && k + 8 * c < K;
            uint4 a[2 * kMmas];
#pragma unroll
            for (int r = 0; r < 2 * kMmas; ++r)
                a[r] = r < ROWS && g + 8 * r < M && in
                           ? __ldg(reinterpret_cast<const uint4 *>(xp + static_cast<int64_t>(8 * r) * K + k))
                           : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int i = 0; i < kMmas; ++i) {
                const uint4 &lo = a[2 * i], &hi = a[2 * i + 1];
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    mma_16816(acc[t][i][0], lo.x, hi.x, lo.y, hi.y, b[t][u].x, b[t][u].y);
                    mma_16816(acc[t][i][1], lo.z, hi.z, lo.w, hi.w, b[t][u].z, b[t][u].w);
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float(&p0)[4] = acc[t][r / 2][0], (&p1)[4] = acc[t][r / 2][1];
            *reinterpret_cast<float2 *>(&part[warp][t][8 * r + g][2 * c]) =
                make_float2(p0[2 * (r & 1)] + p1[2 * (r & 1)], p0[2 * (r & 1) + 1] + p1[2 * (r & 1) + 1]);
        }
    __syncthreads();
    auto out = [&](uint16_t *to, int64_t at, float v) {
        const __nv_bfloat16 b = __float2bfloat16_rn(v);
        to[at] = *reinterpret_cast<const uint16_t *>(&b);
    };
    auto bf = [](uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); };
    const int n = threadIdx.x & 7, col = n0 + n;
    for (int m = threadIdx.x >> 3; m < M; m += WARPS * 4) {
        float f[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f[t] = part[0][t][m][n];
#pragma unroll
            for (int k = 1; k < WARPS; ++k) f[t] += part[k][t][m][n];
        }
        if constexpr (GATED) {
            if (epi.z) {
                out(epi.z, static_cast<int64_t>(m) * 2 * N + col, f[0]);
                out(epi.z, static_cast<int64_t>(m) * 2 * N + N + col, f[kTiles - 1]);
            }
            act_dispatch(epi.act, [&](auto act) { f[0] = act_f32<decltype(act)::value>(f[0]); });
            out(epi.y, static_cast<int64_t>(m) * N + col, f[0] * f[kTiles - 1]);
        } else {
            const int64_t at = static_cast<int64_t>(m) * N + col;
            if (epi.bias) f[0] += bf(epi.bias[col]);
            if (epi.z) out(epi.z, at, f[0]);
            act_dispatch(epi.act, [&](auto act) { f[0] = act_f32<decltype(act)::value>(f[0]); });
            // (y may be the residual: past L1, where a neighbour's part of the sector would stay as it was)
            if (epi.residual) f[0] += bf(__ldcg(epi.residual + m * epi.ld_residual + col));
            out(epi.y, at, f[0]);
        }
    }
}

// (Linears of 17 to 32 tokens: as many blocks of 6 warps as of 8 are resident, of 12 as of 16.)
template <int WARPS, bool GATED, int ROWS>
constexpr bool skinny_built() { return GATED || ROWS < 4 || (WARPS != 6 && WARPS != 12); }

// Blocks of a kernel that are resident at once, cached per device (0: not built, or the query failed, and is asked again).
template <int WARPS, bool GATED, int ROWS>
static int64_t resident_blocks(int dev) {
    if constexpr (!skinny_built<WARPS, GATED, ROWS>()) return 0;
    else {
        static std::atomic<int> cache[64] = {};
        const bool keep = dev >= 0 && dev < 64;
        int n = keep ? cache[dev].load(std::memory_order_relaxed) : 0;
        if (n > 0) return n;
        int per_sm = 0, sms = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, skinny_linear_kernel<WARPS, GATED, ROWS>, WARPS * 32, 0) != cudaSuccess ||
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
            (void)cudaGetLastError();
            return 0;
        }
        n = per_sm * sms;
        if (keep) cache[dev].store(n, std::memory_order_relaxed);
        return n;
    }
}

// Warps a block, which share the reduction: by skinny_form.  One token, us, in a graph,
// at least 400 MB of weights in turn, at 4 / 6 / 8 / 12 / 16 warps: linear [1536] x 8960 (192
// blocks) 33.9 / 23.7 / 14.1 / 14.8 / 7.7, [4096] x 2048 10.2 / 7.5 / 5.3 / 4.9 / 5.5, [8960] x
// 1536 9.1 / 10.2 / 7.2 / 8.2 / 9.3, [9216] x 1536 9.5 / 10.3 / 7.4 / 8.3 / 9.4, [17920] x 1536 16.6 /
// 16.2 / 11.6 / 16.0 / 16.9; gated [1024] x 1024 4.4 / 3.1 / 3.1 / 3.6 / 2.1, [6144] x 2048 14.5 / 12.8
// / 14.4 / 14.2 / 16.0, [8960] x 1536 13.7 / 15.1 / 13.8 / 15.6 / 18.7.  Over 211 widths, reductions
// and numbers of tokens (1 to 32) the rule's choice is 2.1% slower than the fastest of the
// five in the geometric mean and 20% at most ([8192] x 512 on 32 tokens).
template <bool GATED, int ROWS>
static cudaError_t launch_rows(const uint16_t *x, const uint16_t *w, int64_t M, int64_t N, int64_t K, const GemmEpilogue &epi,
                               cudaStream_t s) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int64_t resident[kSkinnyForms] = {resident_blocks<16, GATED, ROWS>(dev), resident_blocks<8, GATED, ROWS>(dev),
                                            resident_blocks<6, GATED, ROWS>(dev), resident_blocks<12, GATED, ROWS>(dev),
                                            resident_blocks<4, GATED, ROWS>(dev)};
    const int warps = kSkinnyWarps[skinny_form(N / 8, (K + 31) / 32, skinny_unroll(GATED), resident)];
    auto kern = warps == 16  ? skinny_linear_kernel<16, GATED, ROWS>
                : warps == 8 ? skinny_linear_kernel<8, GATED, ROWS>
                             : skinny_linear_kernel<4, GATED, ROWS>;
    if constexpr (skinny_built<6, GATED, ROWS>())
        if (warps == 6) kern = skinny_linear_kernel<6, GATED, ROWS>;
    if constexpr (skinny_built<12, GATED, ROWS>())
        if (warps == 12) kern = skinny_linear_kernel<12, GATED, ROWS>;
    return launch_pdl(kern, dim3(static_cast<unsigned>(N / 8)), dim3(warps * 32), 0, s, x, w, static_cast<int>(M),
                      static_cast<int>(N), static_cast<int>(K), epi);
}

// Up to 16 tokens, and up to 32 where the weight is small: every block reads all
// the tokens, from L2, which costs more than the tiles' idle tensor cores where
// there are many blocks.  us here at 17 and 32 tokens / in the GEMM kernel at 33, weights
// out of L2: linear [2048] x 1536 3.9 and 4.2 / 7.8, [2048] x 2048 5.2 and 5.5 / 7.8, [4096] x 1024
// 5.0 and 5.5 / 7.4, gated [1024] x 2048 5.1 and 5.3 / 12.4.  At 16 tokens here / at 33 there:
// [4096] x 2048 7.0 / 8.7, [1536] x 8960 10.1 / 13.0, [8960] x 1536 10.4 / 13.0, but gated [6144] x
// 2048 16.5 / 14.1 and [8960] x 1536 17.0 / 16.3.
bool is_skinny_linear(int64_t M, int64_t N, int64_t K, bool gated) {
    if (K > (1 << 30)) return false;  // (k is an int there)
    return M <= 16 || (M <= 32 && N * K * (gated ? 2 : 1) <= (4 << 20));
}

cudaError_t launch_skinny_linear(const uint16_t *x, const uint16_t *w, int64_t M, int64_t N, int64_t K, bool gated,
                                 const GemmEpilogue &epi, cudaStream_t s) {
    auto launch = M > 16  ? (gated ? launch_rows<true, 4> : launch_rows<false, 4>)
                  : M > 8 ? (gated ? launch_rows<true, 2> : launch_rows<false, 2>)
                          : (gated ? launch_rows<true, 1> : launch_rows<false, 1>);
    return launch(x, w, M, N, K, epi, s);
}

}  // namespace puro
