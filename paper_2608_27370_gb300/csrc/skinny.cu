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

#include "act_math.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "quant_math.cuh"

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

// One block: columns 8 blockIdx.x .. + 7 of the output (GATED: of h, from those
// rows of the gate and of up).  Up to 8 ROWS tokens.
template <int WARPS, bool GATED, int ROWS>
__global__ void __launch_bounds__(WARPS * 32) skinny_linear_kernel(const uint16_t *__restrict__ x, const uint16_t *__restrict__ w,
                                                                  int M, int N, int K, const GemmEpilogue epi) {
    constexpr int kTiles = GATED ? 2 : 1, kUnroll = GATED ? 2 : 3;
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

template <int WARPS, bool GATED>
static cudaError_t launch_warps(const uint16_t *x, const uint16_t *w, int64_t M, int64_t N, int64_t K, const GemmEpilogue &epi,
                                cudaStream_t s) {
    auto kern = M > 16  ? skinny_linear_kernel<WARPS, GATED, 4>
                : M > 8 ? skinny_linear_kernel<WARPS, GATED, 2>
                        : skinny_linear_kernel<WARPS, GATED, 1>;
    return launch_pdl(kern, dim3(static_cast<unsigned>(N / 8)), dim3(WARPS * 32), 0, s, x, w, static_cast<int>(M),
                      static_cast<int>(N), static_cast<int>(K), epi);
}

// Warps a block, which share the reduction: as many as keep the launch within a
// number of warps that are resident at once, since more blocks already spread the
// loads.  One token, us, weights out of L2 in a graph, at 4 / 8 / 16 warps: linear
// [1536] x 8960 (192 blocks) 14.9 / 9.0 / 6.9, [8960] x 1536 (1120 blocks) 7.3 /
// 7.9 / 9.5 (6 warps: 6.2); gated [1024] x 1024 3.2 / 2.5 / 1.9, [8960] x 1536 10.8 /
// 10.7 / 12.5.  Without the prefetch the first takes 10.6 and the last 10.8.
template <bool GATED>
static cudaError_t launch_skinny(const uint16_t *x, const uint16_t *w, int64_t M, int64_t N, int64_t K, const GemmEpilogue &epi,
                                 cudaStream_t s) {
    const int64_t blocks = N / 8, most = GATED ? 9300 : 6800;
    if (blocks * 16 <= most) return launch_warps<16, GATED>(x, w, M, N, K, epi, s);
    if (blocks * 12 <= most) return launch_warps<12, GATED>(x, w, M, N, K, epi, s);
    if (blocks * 8 <= most) return launch_warps<8, GATED>(x, w, M, N, K, epi, s);
    if (blocks * 6 <= most) return launch_warps<6, GATED>(x, w, M, N, K, epi, s);
    return launch_warps<4, GATED>(x, w, M, N, K, epi, s);
}

// Up to 16 tokens, and up to 32 where the weight is small: every block reads all
// the tokens, from L2, which costs more than the tiles' idle tensor cores where
// there are many blocks.  us here / in the GEMM kernel at 17 and 32 tokens: linear
// [2048] x 1536 3.9 / 7.7 and 4.2 / 7.7, [512] x 4096 5.4 / 7.2 and 5.9 / 7.2, but [4096] x
// 2048 9.4 / 8.7 and 10.0 / 8.7, [1536] x 8960 14.2 / 13.8 and 15.9 / 13.9; gated [1024] x
// 1024 2.7 / 8.3 and 2.9 / 8.3, [8960] x 1536 21.7 / 15.9 and 22.9 / 15.7 (at 16 tokens
// 15.2 / 15.9).
bool is_skinny_linear(int64_t M, int64_t N, int64_t K, bool gated) {
    if (K > (1 << 30)) return false;  // (k is an int there)
    return M <= 16 || (M <= 32 && N * K * (gated ? 2 : 1) <= (4 << 20));
}

cudaError_t launch_skinny_linear(const uint16_t *x, const uint16_t *w, int64_t M, int64_t N, int64_t K, bool gated,
                                 const GemmEpilogue &epi, cudaStream_t s) {
    return gated ? launch_skinny<true>(x, w, M, N, K, epi, s) : launch_skinny<false>(x, w, M, N, K, epi, s);
}

}  // namespace puro
