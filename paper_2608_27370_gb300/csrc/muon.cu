// muon.cu -- the Muon directions u of many matrices: the momentum's update, and its
// orthogonalisation by Newton-Schulz products (Puro-2B, section "Hyperball
// Optimization", takes the Muon update direction u as given and does not specify
// the orthogonalisation; this is the published one: odd polynomials of the update's
// singular values, a few products each).
//
// For a matrix of m x n, m <= n (a taller one is transposed on its way in and out):
//     V = the momentum's update,  X = V / ||V||_F,
//     per step (a, b, c):  A = X X^T,  X <- (a I + b A + c A^2) X.
//
// How it is computed here.  The products run on the tensor cores in FP16 with FP32
// accumulation (FP16 for its 11 digits: the singular values are at most about one,
// so that a power of two per step puts every matrix in range).  Two steps at a time,
// with G = X X^T, B0 = a I + b G + c G^2:
//     G1 = B0 G B0 (the next step's G, for B0 and G commute),
//     B1 = a' I + b' G1 + c' G1^2,  X <- (B1 B0) X,
// so that products of m x m take the place of the second step's two of m x n: for n =
// 6 m a pair of steps takes 12.5 m^3 products and sums for 19.  G, B0, G1 and B1 are
// symmetric: computed on and above the diagonal and stored twice.
//
// Where digits are lost.  A rounding of X adds noise of full rank, and the steps
// blow small singular values up (3.4 times each, by Muon's coefficients), the noise
// with them, the first rounding the most; a rounding of B only turns X's rows a little
// into one another.  So the first X is two FP16 numbers, x = hi + lo, scaled to a norm of
// about 2^9 (2^6 to 2^16): 22 digits of the larger values, the rest to half of FP16's
// least step, 2^-25 (values of [8960, 1536] are 0.14 on average at 2^9: 22 digits, at the
// least norm 19).  B1 B0 multiplies both (lo after hi, into the same accumulator), and G
// takes hi alone.  A
// rounding of G is harmless in B0 but blown up in G1, so behind the first pair G, too, is
// hi + lo for G1.  And G1 is B0 (B0 G)^T, symmetric whatever B0's roundings: as (B0 G) B0
// with a mirrored or transposed factor it doubles the error, for rounded B0 and G no
// longer commute.  u is then off by 1.0 to 1.9 10^-3 of its 2-norm for momenta of rank 16
// and noise half as large, 48 x 80 to 2048 x 6144 (G without lo: up to 2.0; every BF16
// operand: eight times as much).  Where the noise is 1/130 of a signal of rank 16, by
// 7 10^-3 (X without lo: 20; lo of the second pair's X, too: 2, for a fifth of the time
// more).
//
// Measured and not kept: all products in one cooperative launch with a barrier of all
// blocks between them (one [1536, 1536] 205 us for 178, a layer of Qwen2-1.5B 1162 for
// 1142), and as tickets that pairs draw, each tile waiting for its matrix's product before
// (207 for 177, 965 for 990); two CTAs of narrow tiles an SM (191 for 177).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <memory>
#include <new>
#include <type_traits>

#include "internal.h"
#include "muon_plan.h"
#include "ptx.cuh"

namespace puro {
namespace {

constexpr int kMaxSteps = 64;
constexpr int32_t kStatusTimeout = 4;  // PURO_ERR_TIMEOUT
constexpr uint64_t kDrainNs = 2000000000ull, kSettleNs = 200000ull;

// ------------------------------------------------ the update and its norm
constexpr int kInRows = 64, kInCols = 128, kInThreads = 256;  // tile of the two passes over V
constexpr int kInWarps = kInThreads / 32, kInPasses = 4;  // a warp a row, four rows of a warp at a time

enum MatFlags : uint8_t {
    kGradBf16 = 1,
    kTall = 2,      // more rows than columns: X is its transpose
    kVectors = 4,   // four columns of a row can be read at once in momentum (and stored in X)
    kOutF32 = 8,
    kGradVectors = 32,  // and in grad
    kOutVectors = 16,  // eight columns of a row of u can be stored in 16-byte pieces
};
// How X is held ahead of the first step: hi + lo is guess V (a power of two that a
// sample of the gradient gave), and r of it is X; or, where that would have left
// FP16's range, hi + lo is V x y = 2^14 X.
struct MuonScale {
    float r, x, y;
};
// One matrix's part of the update (together: a block's first use of a parameter is a
// cache miss).
struct alignas(16) MatIn {
    const void *grad;
    float *momentum;
    int64_t stride;
    uint16_t *hi, *lo;
    int rows, cols, ldx;
    uint8_t flags;
};
struct MuonIn {
    int count;
    float mu;
    int nesterov;
    bool store_lo;
    double *partial;  // [tiles]: sum of V^2 over each
    float *guess;      // [count]
    MuonScale *scale;  // [count]
    int tile0[kMaxMats + 1];  // first tile of each matrix
    MatIn mat[kMaxMats];
};

PURO_DEV int mat_of(const int *start, int count, int t) {
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// A lane's four columns of a tile's row: neighbours where grad and momentum can be
// read in vectors, else 32 apart, so that a warp's accesses are dense either way.
PURO_DEV int in_col(uint8_t flags, int lane, int k) { return flags & kVectors ? 4 * lane + k : lane + 32 * k; }

// The values of V of a lane's columns c0 ... in rows r0 + warp, r0 + warp + kInWarps, ...,
// zero outside the matrix.  UPDATE: the momentum takes the gradient first and is
// stored; else it has.  All loads are issued ahead of the first use (with each row's
// behind the row before's stores 114 us for 82 over a layer's matrices); what is read
// once makes room in L2 for X first.
template <bool UPDATE, bool VEC, bool GRAD_VEC, bool BF16>
PURO_DEV void tile_of(const MuonIn &p, int m, int r0, int c0, float (&v)[kInPasses][4]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rows = p.mat[m].rows, cols = p.mat[m].cols;
    float *const mom = p.mat[m].momentum;
    const bool read_g = UPDATE || !mom || p.nesterov;
    const int64_t stride = p.mat[m].stride;
    float w[kInPasses][4];
    auto in = [&](int i, int k) { return r0 + warp + kInWarps * i < rows && c0 + (VEC ? 4 * lane : lane + 32 * k) < cols; };
    auto at = [&](int i, int k, int64_t pitch) { return (r0 + warp + kInWarps * i) * pitch + c0 + (VEC ? 4 * lane : lane + 32 * k); };
#pragma unroll
    for (int i = 0; i < kInPasses; ++i) {
        if constexpr (VEC) {
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (in(i, 0)) {
                if (read_g) {
                    if constexpr (!GRAD_VEC) {  // (a warp's loads of one k are 8 or 16 bytes apart: the next find them in L1)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int64_t from = at(i, 0, stride) + k;
                            const uint32_t z = BF16 ? __ldg(static_cast<const uint16_t *>(p.mat[m].grad) + from)
                                                    : __float_as_uint(__ldg(static_cast<const float *>(p.mat[m].grad) + from));
                            if (BF16)
                                (k < 2 ? x.x : x.y) |= z << (16 * (k & 1));
                            else
                                (k == 0 ? x.x : k == 1 ? x.y : k == 2 ? x.z : x.w) = z;
                        }
                    } else if constexpr (BF16) {
                        const uint2 z = __ldcs(reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p.mat[m].grad) + at(i, 0, stride)));
                        x.x = z.x;
                        x.y = z.y;
                    } else {
                        x = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const float *>(p.mat[m].grad) + at(i, 0, stride)));
                    }
                }
                if (mom) y = __ldcs(reinterpret_cast<const float4 *>(mom + at(i, 0, cols)));
            }
            v[i][0] = __uint_as_float(BF16 ? x.x << 16 : x.x);
            v[i][1] = __uint_as_float(BF16 ? x.x & 0xFFFF0000u : x.y);
            v[i][2] = __uint_as_float(BF16 ? x.y << 16 : x.z);
            v[i][3] = __uint_as_float(BF16 ? x.y & 0xFFFF0000u : x.w);
            w[i][0] = y.x;
            w[i][1] = y.y;
            w[i][2] = y.z;
            w[i][3] = y.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[i][k] = w[i][k] = 0.0f;
                if (!in(i, k)) continue;
                if (read_g)
                    v[i][k] = BF16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(p.mat[m].grad)[at(i, k, stride)]) << 16)
                                   : static_cast<const float *>(p.mat[m].grad)[at(i, k, stride)];
                if (mom) w[i][k] = mom[at(i, k, cols)];
            }
        }
    }
    if (!mom) return;
    if constexpr (UPDATE) {
#pragma unroll
        for (int i = 0; i < kInPasses; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[i][k] = fmaf(p.mu, w[i][k], v[i][k]);
            if constexpr (VEC) {
                if (in(i, 0)) __stcs(reinterpret_cast<float4 *>(mom + at(i, 0, cols)), make_float4(w[i][0], w[i][1], w[i][2], w[i][3]));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (in(i, k)) mom[at(i, k, cols)] = w[i][k];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kInPasses; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i][k] = p.nesterov ? fmaf(p.mu, w[i][k], v[i][k]) : w[i][k];
}
template <bool UPDATE>
PURO_DEV void read_tile(const MuonIn &p, int m, int r0, int c0, float (&v)[kInPasses][4]) {
    const uint8_t f = p.mat[m].flags;
    auto read = [&](auto bf16) {
        constexpr bool kBf16 = decltype(bf16)::value;
        if (!(f & kVectors))
            tile_of<UPDATE, false, false, kBf16>(p, m, r0, c0, v);
        else if (f & kGradVectors)
            tile_of<UPDATE, true, true, kBf16>(p, m, r0, c0, v);
        else
            tile_of<UPDATE, true, false, kBf16>(p, m, r0, c0, v);
    };
    if (f & kGradBf16)
        read(std::true_type{});
    else
        read(std::false_type{});
}

// The lines that a warp reads of half a tile at (r0, c0), to L2: one to a lane.
PURO_DEV void prefetch_half(const MuonIn &p, int m, int r0, int c0) {
    const int lane = threadIdx.x & 31, i = (lane >> 2) & 3, c = c0 + 32 * (lane & 3);
    const int r = r0 + (threadIdx.x >> 5) + kInWarps * i;
    if (r >= p.mat[m].rows || c >= p.mat[m].cols) return;
    const void *at;
    if (lane < 16)
        at = p.mat[m].flags & kGradBf16 ? static_cast<const void *>(static_cast<const uint16_t *>(p.mat[m].grad) + r * p.mat[m].stride + c)
                                        : static_cast<const float *>(p.mat[m].grad) + r * p.mat[m].stride + c;
    else if (p.mat[m].momentum)
        at = p.mat[m].momentum + static_cast<int64_t>(r) * p.mat[m].cols + c;
    else
        return;
    prefetch_l2(at);
}

struct InTile {
    int r0, c0;
};
PURO_DEV InTile in_tile(int i, int cols) {
    const int across = (cols + kInCols - 1) / kInCols;
    return {i / across * kInRows, i % across * kInCols};
}

PURO_DEV double warp_sum(double d) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xFFFFFFFFu, d, o);
    return d;
}

// hi + lo of v scaled, four values of a row of the tile at (r0, c0): to X, or for a tall
// matrix to `turn`, which store_turned() writes.  turn[c][r ^ (c / 4) % 32]: without
// bank conflicts for lanes that hold four neighbouring columns.
struct Turn {
    uint32_t at[kInCols][kInRows];
};
PURO_DEV void store_x(const MuonIn &p, int m, Turn &turn, int r0, int lr, int c0, const float (&v)[4], float f0, float f1) {
    const uint8_t flags = p.mat[m].flags;
    const int lane = threadIdx.x & 31, ldx = p.mat[m].ldx, r = r0 + lr;
    uint32_t x[4];  // hi, lo
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float y = (v[k] * f0) * f1;
        const __half h = __float2half_rn(y), l = __float2half_rn(y - __half2float(h));
        x[k] = __half_as_ushort(h) | static_cast<uint32_t>(__half_as_ushort(l)) << 16;
    }
    if (flags & kTall) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = in_col(flags, lane, k);
            turn.at[c][lr ^ ((flags & kVectors ? c >> 2 : c) & 31)] = x[k];
        }
    } else if (r < p.mat[m].rows) {
        const int64_t at = static_cast<int64_t>(r) * ldx + c0;
        if (flags & kVectors) {
            if (c0 + 4 * lane >= ldx) return;
            *reinterpret_cast<uint2 *>(p.mat[m].hi + at + 4 * lane) = make_uint2(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410));
            if (p.store_lo)
                *reinterpret_cast<uint2 *>(p.mat[m].lo + at + 4 * lane) = make_uint2(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = lane + 32 * k;
                if (c0 + c >= ldx) continue;
                p.mat[m].hi[at + c] = static_cast<uint16_t>(x[k]);
                if (p.store_lo) p.mat[m].lo[at + c] = static_cast<uint16_t>(x[k] >> 16);
            }
        }
    }
}
// A row of X is a column of V: 64 values, two to a lane.
PURO_DEV void store_turned(const MuonIn &p, int m, const Turn &turn, int r0, int c0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ldx = p.mat[m].ldx, r = r0 + 2 * lane;
    const bool vec = p.mat[m].flags & kVectors;
    if (r >= ldx) return;
#pragma unroll 4
    for (int c = warp; c < kInCols; c += kInWarps) {
        if (c0 + c >= p.mat[m].cols) break;
        const int turned = (vec ? c >> 2 : c) & 31;
        const uint32_t a = turn.at[c][(2 * lane) ^ turned], b = turn.at[c][(2 * lane + 1) ^ turned];
        const int64_t at = static_cast<int64_t>(c0 + c) * ldx + r;
        *reinterpret_cast<uint32_t *>(p.mat[m].hi + at) = __byte_perm(a, b, 0x5410);
        if (p.store_lo) *reinterpret_cast<uint32_t *>(p.mat[m].lo + at) = __byte_perm(a, b, 0x7632);
    }
}

constexpr int kSampled = 1024;      // values of the gradient that the guess goes by
constexpr int kGuessExp = 9;        // it puts their norm's estimate at 2^9: V's may be 2^7 times that, or 2^-3
constexpr double kLeastNorm = 64.0, kMostNorm = 65024.0;  // what guess ||V|| has to lie in: FP16's largest value is 65504

// The momentum takes the gradient; each tile's sum of V^2; hi + lo of V times a power
// of two.  V is not read again for that (12 bytes a value of 28), so the factor has to
// be known before the norm: each block takes it from the same sample of the gradient,
// and muon_norm_kernel finds whether it holds.  A thread's 16 squares of half a tile
// and its warp's are summed in FP32, in FP64 where that left its range; the warps' and
// tiles' in FP64 in a fixed order.  Bound by memory: a block has a run of tiles, all
// blocks equally many, across the matrices, and asks L2 for half a tile ahead (a sum for
// each of at most 256 runs of a matrix's tiles had left the large ones 1.6 blocks an SM;
// a call for Qwen2-1.5B's layer took 996 us so, 965 with the blocks level;
// 24 matrices of [128, 1536] and 11 small ones 157 and 145).
__global__ void __launch_bounds__(kInThreads, 4) muon_update_kernel(const __grid_constant__ MuonIn p) {
    __shared__ Turn turn;
    __shared__ double part[2][kInWarps];
    __shared__ float sampled[kInWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int64_t all = p.tile0[p.count];
    const int end = static_cast<int>(all * (blockIdx.x + 1) / gridDim.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int i = static_cast<int>(all * blockIdx.x / gridDim.x);
    for (int m = mat_of(p.tile0, p.count, i); i < end; ++m) {
        const bool tall = p.mat[m].flags & kTall;
        float sample = 0.0f;  // rows evenly, columns by a hash
#pragma unroll
        for (int j = 0; j < kSampled / kInThreads; ++j) {
            const uint32_t e = threadIdx.x + kInThreads * j;
            const int64_t at = (e * static_cast<uint32_t>(p.mat[m].rows) / kSampled) * p.mat[m].stride +
                               __umulhi(e * 2654435761u, static_cast<uint32_t>(p.mat[m].cols));
            sample += fabsf(p.mat[m].flags & kGradBf16
                                ? __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t *>(p.mat[m].grad) + at)) << 16)
                                : __ldg(static_cast<const float *>(p.mat[m].grad) + at));
        }
        float guess = 0.0f;
        for (const int last = min(end, p.tile0[m + 1]); i < last; ++i) {
            const InTile t = in_tile(i - p.tile0[m], p.mat[m].cols);
            float sum = 0.0f;
            double far = 0.0;  // what FP32 does not hold
#pragma unroll 1
            for (int half = 0; half < kInRows; half += kInWarps * kInPasses) {
                float v[kInPasses][4], s = 0.0f, most = 0.0f;
                read_tile<true>(p, m, t.r0 + half, t.c0, v);
                if (half == 0) {
                    prefetch_half(p, m, t.r0 + kInWarps * kInPasses, t.c0);
                } else if (i + 1 < last) {
                    const InTile next = in_tile(i + 1 - p.tile0[m], p.mat[m].cols);
                    prefetch_half(p, m, next.r0, next.c0);
                }
                if (guess == 0.0f) {  // once a matrix, beside the first reads
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sample += __shfl_xor_sync(0xFFFFFFFFu, sample, o);
                    if (lane == 0) sampled[warp] = sample;
                    __syncthreads();
                    float n = 0.0f;
#pragma unroll
                    for (int w = 0; w < kInWarps; ++w) n += sampled[w];
                    // ||g|| is about the mean of |g| times sqrt(total)
                    n *= (1.0f / kSampled) * sqrtf(static_cast<float>(p.mat[m].rows) * static_cast<float>(p.mat[m].cols));
                    const int k = n > 0.0f && n < INFINITY ? min(max(kGuessExp - ilogbf(n), -126), 127) : 0;
                    guess = __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
                    if (i == p.tile0[m] && threadIdx.x == 0) p.guess[m] = guess;
                }
#pragma unroll
                for (int j = 0; j < kInPasses; ++j) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        s = fmaf(v[j][k], v[j][k], s);
                        most = fmaxf(most, fabsf(v[j][k]));
                    }
                    store_x(p, m, turn, t.r0, half + warp + kInWarps * j, t.c0, v[j], guess, 1.0f);
                }
                if (s > 1e-24f && s < 1e36f) {
                    sum += s;
                } else if (!(s == 0.0f && most == 0.0f)) {  // (FP64 is 64 times slower: not for what lies outside the matrix)
#pragma unroll
                    for (int j = 0; j < kInPasses; ++j)
#pragma unroll
                        for (int k = 0; k < 4; ++k) far += static_cast<double>(v[j][k]) * v[j][k];
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            double *const parts = part[i & 1];  // the tile before's are still read
            const bool any = __any_sync(0xFFFFFFFFu, far != 0.0);
            if (any) far = warp_sum(far);
            if (lane == 0) parts[warp] = any ? sum + far : sum;
            __syncthreads();
            if (threadIdx.x == 0) {
                double d = 0.0;
#pragma unroll
                for (int w = 0; w < kInWarps; ++w) d += parts[w];
                p.partial[i] = d;
            }
            if (tall) {
                store_turned(p, m, turn, t.r0, t.c0);
                __syncthreads();
            }
        }
    }
}

// The first X's power of two where the guess did not hold: entries are at most 1.
constexpr int kX0Exp = 14;

// Each matrix's norm, and by it what the first step multiplies with: NaN where it is
// not finite (all of u is then NaN), 0 for V = 0.  And X once more where the guess did not
// hold.  Block (b, m) of gridDim.x for matrix m; each adds the norm up for itself, which
// is a launch less than to be told (one [48, 80] 42.6 -> 40.1 us, [1536, 1536] 171.9 -> 169.3).
__global__ void __launch_bounds__(kInThreads, 3) muon_norm_kernel(const __grid_constant__ MuonIn p) {
    __shared__ Turn turn;
    __shared__ double part[kInWarps];
    __shared__ MuonScale again;  // what X is written with once more, or 0
    constexpr int kAtOnce = 16;
    pdl_wait();
    pdl_launch_dependents();
    const int m = blockIdx.y, first = p.tile0[m], end = p.tile0[m + 1], warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (8 * static_cast<int>(blockIdx.x) >= end - first) return;
    double d = 0.0;
    for (int i = first + 32 * warp; i < end; i += kAtOnce * kInThreads) {  // (few additions: FP64 is 64 times slower)
        double v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) v[j] = j * kInThreads + lane < end - i ? p.partial[i + j * kInThreads + lane] : 0.0;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (j * kInThreads < end - i) d += v[j];
    }
    if (first + 32 * warp < end) d = warp_sum(d);
    if (lane == 0) part[warp] = d;
    __syncthreads();
    if (warp == 0) {
        d = part[0];
#pragma unroll
        for (int w = 1; w < kInWarps; ++w)
            if (first + 32 * w < end) d += part[w];
        const float guess = p.guess[m];
        MuonScale s{0.0f, 0.0f, 0.0f};
        bool redo = false;
        if (!(d < INFINITY)) {
            s.r = NAN;
        } else if (d > 0.0) {
            const double held2 = d * guess * guess;
            redo = !(held2 >= kLeastNorm * kLeastNorm && held2 <= kMostNorm * kMostNorm);
            if (!redo) {
                if (blockIdx.x == 0) s.r = static_cast<float>(1.0 / (sqrt(d) * guess));
            } else {
                // the factor in two parts, neither of which leaves FP32's range
                const double scale = static_cast<double>(1 << kX0Exp) / sqrt(d);
                const int e = ilogb(scale) / 2;
                s.x = static_cast<float>(ldexp(1.0, e));
                s.y = static_cast<float>(ldexp(scale, -e));
                s.r = 1.0f / static_cast<float>(1 << kX0Exp);
            }
        }
        if (blockIdx.x == 0 && lane == 0) p.scale[m] = s;
        if (lane == 0) again = redo ? s : MuonScale{0.0f, 0.0f, 0.0f};
    }
    __syncthreads();
    const MuonScale s = again;
    if (s.x == 0.0f) return;
    const int blocks = min(static_cast<int>(gridDim.x), (end - first + 7) / 8);
    for (int i = blockIdx.x; i < end - first; i += blocks) {
        const InTile t = in_tile(i, p.mat[m].cols);
#pragma unroll 1
        for (int half = 0; half < kInRows; half += kInWarps * kInPasses) {
            float v[kInPasses][4];
            read_tile<false>(p, m, t.r0 + half, t.c0, v);
#pragma unroll
            for (int j = 0; j < kInPasses; ++j) store_x(p, m, turn, t.r0, half + warp + kInWarps * j, t.c0, v[j], s.x, s.y);
        }
        if (p.mat[m].flags & kTall) {
            __syncthreads();
            store_turned(p, m, turn, t.r0, t.c0);
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------ the products
// D = A B^T in FP16 (kind::f16), FP32 accumulators, as CTA pairs compute the linears'
// products (see gemm.cu): pair MMAs of 256 x BN, a ring of k-blocks of 64 that the
// TMA fills, two accumulators, so that a tile's epilogue runs beside the next one's
// MMAs.
//   warp 0       TMA producer (both CTAs)
//   warp 1       MMA issuer (even CTA); tensor memory
//   warps 4..11  epilogue (both CTAs): warp 4 + 4h + q has rows 32q .. of the CTA's
//                128 and the h-th half of the columns
// B is [N, K] with K contiguous, or X_MAJOR [K, N] with N contiguous (X as the right
// factor of B X), which the tensor cores read as it lies (MN-major).  The matrices
// of one shape are a class: one tensor map each for A, B and D with the matrix as
// the third coordinate.
constexpr int kBM = 128;
constexpr int kThreads = 384;
constexpr int kEpiWarps = 8;
constexpr int kTmemCols = 512;

enum Epilogue : int {
    kStore = 0,  // alpha D as hi (and lo), symmetric
    kPoly = 1,   // alpha D + beta G + gamma I, symmetric
    kNext = 2,   // alpha D as hi (and lo)
    kOut = 3,    // alpha D to u
};

struct MuonMaps {
    CUtensorMap a, a_lo, b, b_lo, d, d_lo;  // a: box 64 x 128; b: 64 x BN / 2, X_MAJOR 64 x 64; d: 32 x 32 (64-byte swizzle)
};
struct MuonPhase : Tiles {
    MuonMaps maps[kMaxClasses];
    int passes[kMaxClasses];     // over A and B: 2, B's lo after its hi; 3, then A's lo with B's hi
    bool store_lo[kMaxClasses];
    const uint16_t *g[kMaxClasses], *g_lo[kMaxClasses];  // kPoly: G of the first matrix, and its lo or null
    int64_t g_batch[kMaxClasses];
    int ldg[kMaxClasses];
    float alpha, beta, gamma;
    const MuonScale *scale;      // of the first X, or null: alpha times r, of X X^T r^2
    bool squared;
    uint32_t idesc;
    int32_t *status;
    uint64_t wait_ns;
};
struct MuonOut {
    void *u[kMaxMats];
    int64_t stride[kMaxMats];
    uint8_t flags[kMaxMats];
};
struct NoOut {};
template <int EPI>
using OutOf = std::conditional_t<EPI == kOut, MuonOut, NoOut>;  // (launches copy their parameters)

template <int BN>
struct ProductSmem {
    static constexpr int kStages = 192 * 1024 / (kBM * 128 + BN / 2 * 128);  // 6 (256), 8 (128)
    alignas(1024) uint8_t a[kStages][kBM * 128];
    alignas(1024) uint8_t b[kStages][BN / 2 * 128];
    alignas(1024) uint8_t stage[kEpiWarps][4096];
    uint64_t full[kStages], empty[kStages];
    uint64_t tfull[2], tempty[2];
    uint64_t drain;
    uint32_t tmem_base;
    volatile int abort_flag;
};
template <class Smem>
PURO_DEV bool wait_or_abort(Smem &sm, uint64_t *bar, uint32_t parity, uint64_t ns, int32_t *status, int lane) {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity)) ||
        __all_sync(0xFFFFFFFFu, sm.abort_flag == 0 && mbar_wait_bounded(bar, parity, ns)))
        return true;
    if (lane == 0) {
        sm.abort_flag = 1;
        if (status) atomicExch(status, kStatusTimeout);
    }
    return false;
}

PURO_DEV uint32_t half2_bits(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
PURO_DEV uint32_t bf162_bits(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// A 32 x 32 block of 16-bit values in the staging tile, rows of 64 bytes with the
// 64-byte swizzle; w holds the lane's row in pairs of columns.
PURO_DEV void stage_rows(uint8_t *to, const uint32_t (&w)[16], int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint4 *>(to + 64 * lane + 16 * (i ^ ((lane >> 1) & 3))) =
            make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
// Its transpose: the lane's row becomes a column.  Neighbouring lanes exchange
// halves, so that each stores two rows' values of one column in 32 bits.
PURO_DEV void stage_columns(uint8_t *to, const uint32_t (&w)[16], int lane) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {  // columns 2i (even lanes) and 2i + 1 (odd lanes)
        const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, w[i], 1);
        const uint32_t x = lane & 1 ? __byte_perm(other, w[i], 0x7632) : __byte_perm(w[i], other, 0x5410);
        const int row = 2 * i + (lane & 1), word = lane >> 1;
        *reinterpret_cast<uint32_t *>(to + 64 * row + 16 * ((word >> 2) ^ ((row >> 1) & 3)) + 4 * (word & 3)) = x;
    }
}

// A staged block to rows r0 .. and columns c0 .. of u.
PURO_DEV void block_to_u(const uint8_t *from, bool f32, bool vectors, void *u, int64_t stride, int r0, int c0, int rows, int cols,
                         int lane) {
    if (vectors) {
        const int per = f32 ? 8 : 4;  // 16-byte pieces of a row
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = (32 / per) * i + lane / per, piece = lane % per;
            if (row >= 32) break;
            const int c = c0 + piece * (32 / per);
            if (r0 + row >= rows || c >= cols) continue;
            const int s = f32 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3);
            const uint4 x = *reinterpret_cast<const uint4 *>(from + (f32 ? 128 : 64) * row + 16 * s);
            const int64_t at = (r0 + row) * stride + c;
            *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(u) + at * (f32 ? 4 : 2)) = x;
        }
        return;
    }
    if (c0 + lane >= cols) return;
    for (int row = 0; row < 32 && r0 + row < rows; ++row) {
        const int64_t at = (r0 + row) * stride + c0 + lane;
        if (f32)
            static_cast<float *>(u)[at] = *reinterpret_cast<const float *>(from + 128 * row + 16 * ((lane >> 2) ^ (row & 7)) + 4 * (lane & 3));
        else
            static_cast<uint16_t *>(u)[at] =
                *reinterpret_cast<const uint16_t *>(from + 64 * row + 16 * ((lane >> 3) ^ ((row >> 1) & 3)) + 2 * (lane & 7));
    }
}

// A lane's row of 32 x 32 values at (row0, col) of X, of rows x cols, to u.
PURO_DEV void values_to_u(uint8_t *stage, const MuonOut &out, int m, const float (&v)[32], int row0, int col, int rows, int cols,
                          int lane) {
    const uint8_t f = out.flags[m];
    const bool tall = f & kTall, f32 = f & kOutF32;
    __syncwarp();  // the block before has left the staging tile
    if (f32) {
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const int sr = tall ? k : lane, sc = tall ? lane : k;
            *reinterpret_cast<float *>(stage + 128 * sr + 16 * ((sc >> 2) ^ (sr & 7)) + 4 * (sc & 3)) = v[k];
        }
    } else {
        uint32_t h[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) h[k] = bf162_bits(v[2 * k], v[2 * k + 1]);
        if (tall)
            stage_columns(stage, h, lane);
        else
            stage_rows(stage, h, lane);
    }
    __syncwarp();
    block_to_u(stage, f32, f & kOutVectors, out.u[m], out.stride[m], tall ? col : row0, tall ? row0 : col, tall ? cols : rows,
               tall ? rows : cols, lane);
}

template <int BN, bool X_MAJOR, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    muon_product_kernel(const __grid_constant__ MuonPhase p, const __grid_constant__ OutOf<EPI> out) {
    using Smem = ProductSmem<BN>;
    constexpr int kStages = Smem::kStages;
    constexpr bool kSym = EPI == kStore || EPI == kPoly;
    constexpr int kWarpCols = BN / 2;                           // columns of an epilogue warp
    constexpr uint32_t kStageBytes = kBM * 128 + BN / 2 * 128;  // of one CTA
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = __shfl_sync(0xFFFFFFFFu, static_cast<int>(cluster_ctarank()), 0);
    const int pair = blockIdx.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.tfull[b], 1);
            mbar_init(&sm.tempty[b], 2 * kEpiWarps);
        }
        mbar_init(&sm.drain, 1);
        sm.abort_flag = 0;
        fence_mbarrier_init();
    }
    __syncthreads();
    if (warp == 1) {
        tmem_alloc_pair(&sm.tmem_base, kTmemCols);
        tmem_relinquish_alloc_permit_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    cluster_arrive();
    cluster_wait();  // both CTAs' barriers exist
    const uint32_t tmem = sm.tmem_base;
    // The first unit is worked out, and its maps fetched, before the wait for the kernel
    // before (the empty asm keeps it there).
    Walk walk;
    int u = walk.next(p, pair);
    Unit w{};
    if (u >= 0) w = unit_of<BN, kSym>(p, u);
    asm volatile("" : "+r"(w.cls), "+r"(w.z), "+r"(w.m0), "+r"(w.n0), "+r"(w.kb));
    auto next = [&] {
        u = walk.next(p, pair);
        if (u >= 0) w = unit_of<BN, kSym>(p, u);
    };

    if (warp == 0) {
        // ------------------------------------------------ TMA producer
        const uint32_t e = elect_one();
        const uint32_t full0 = mapa_shared(smem_u32(&sm.full[0]), 0);
        uint32_t stage = 0, phase = 0, issued = 0;
        bool ok = true;
        if (lane < 3 + (EPI == kOut ? 0 : 1)) {
            const MuonMaps &m = p.maps[w.cls];
            tma_prefetch_desc(lane == 0 ? &m.a : lane == 1 ? &m.b : lane == 2 && p.passes[w.cls] > 1 ? &m.b_lo : lane == 3 ? &m.d : &m.a);
        }
        __syncwarp();
        pdl_wait();
        pdl_launch_dependents();
        for (; u >= 0 && ok; next()) {
            const MuonMaps &maps = p.maps[w.cls];
            const int a_row = w.m0 + kBM * rank, b_row = w.n0 + BN / 2 * rank;
            for (int pass = 0; pass < p.passes[w.cls] && ok; ++pass) {
                const CUtensorMap *ma = pass == 2 ? &maps.a_lo : &maps.a, *mb = pass == 1 ? &maps.b_lo : &maps.b;
                for (int kb = 0; kb < w.kb; ++kb) {
                    ok = wait_or_abort(sm, &sm.empty[stage], phase ^ 1u, p.wait_ns, p.status, lane);
                    if (!ok) break;
                    const uint32_t bar = full0 + 8u * stage;
                    if (rank == 0 && e) mbar_arrive_expect_tx(&sm.full[stage], 2u * kStageBytes);
                    tma_load_3d_pair_e(e, sm.a[stage], ma, bar, kb * kBK, a_row, w.z);
                    if constexpr (X_MAJOR) {
#pragma unroll
                        for (int i = 0; i < BN / 128; ++i)
                            tma_load_3d_pair_e(e, sm.b[stage] + 8192 * i, mb, bar, b_row + 64 * i, kb * kBK, w.z);
                    } else {
                        tma_load_3d_pair_e(e, sm.b[stage], mb, bar, kb * kBK, b_row, w.z);
                    }
                    ++issued;
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
        if (rank == 0) {  // every fill of the ring (both CTAs' copies) lands before the pair exits
            for (uint32_t s = 0; s < kStages; ++s) {
                const uint32_t fills = issued / kStages + (s < issued % kStages ? 1u : 0u);
                if (fills > 0) mbar_wait_bounded(&sm.full[s], (fills - 1u) & 1u, kDrainNs);
            }
        }
        if (!ok) {  // this CTA's copies count on the even CTA's barriers: give those in flight time to land
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < kSettleNs) {
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------ MMA issuer
        const uint32_t e = elect_one();
        uint32_t stage = 0, phase = 0;
        int local = 0;
        bool ok = true;
        for (; u >= 0 && ok; next(), ++local) {
            const int buf = local & 1;
            ok = wait_or_abort(sm, &sm.tempty[buf], ((local >> 1) & 1u) ^ 1u, p.wait_ns, p.status, lane);
            if (local == 0) pdl_wait();  // (the kernel before is not what a bounded wait is for)
            const uint32_t d = tmem + static_cast<uint32_t>(BN) * buf;
            const int kbs = w.kb * p.passes[w.cls];
            for (int kb = 0; kb < kbs && ok; ++kb) {
                ok = wait_or_abort(sm, &sm.full[stage], phase, p.wait_ns, p.status, lane);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t a = smem_u32(sm.a[stage]), b = smem_u32(sm.b[stage]);
#pragma unroll
                for (int k = 0; k < kBK / 16; ++k) {
                    const uint64_t bd = X_MAJOR ? smem_desc_mn_sw128(b + 2048 * k, 8192) : smem_desc_k_sw128(b + 32 * k);
                    mma_pair_f16_e(e, d, smem_desc_k_sw128(a + 32 * k), bd, p.idesc, kb > 0 || k > 0 ? 1u : 0u);
                }
                tc_commit_pair_multicast_e(e, &sm.empty[stage], 3);
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (ok) tc_commit_pair_multicast_e(e, &sm.tfull[buf], 3);
        }
        if (e) {  // all MMAs issued are complete before teardown
            tc_commit_pair(&sm.drain);
            mbar_wait_bounded(&sm.drain, 0, kDrainNs);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) >> 2;
        const uint32_t e = elect_one();
        uint8_t *stage_buf = sm.stage[warp - 4];
        const uint32_t tempty0 = mapa_shared(smem_u32(&sm.tempty[0]), 0);
        uint32_t pieces = 0;
        // one 32 x 32 block by way of the next half of the staging tile
        auto store = [&](const CUtensorMap *map, const uint32_t(&w)[16], bool transposed, int x, int y, int z) {
            uint8_t *to = stage_buf + 2048 * (pieces & 1u);
            if (e) bulk_wait_group_read<1>();
            __syncwarp();
            if (transposed)
                stage_columns(to, w, lane);
            else
                stage_rows(to, w, lane);
            fence_proxy_async_smem();
            __syncwarp();
            tma_store_3d_e(e, map, to, x, y, z);
            ++pieces;
        };
        int local = 0;
        pdl_wait();  // (before G is read and anything stored)
        for (; u >= 0; next(), ++local) {
            const int buf = local & 1;
            const MuonMaps &maps = p.maps[w.cls];
            const int row0 = w.m0 + kBM * rank + 32 * q, rows = p.rows[w.cls], cols = p.cols[w.cls];
            float alpha = p.alpha;
            if (p.scale) {
                const float x = __ldg(&p.scale[p.first[w.cls] + w.z].r);
                alpha *= p.squared ? x * x : x;
            }
            uint4 g[4];
            auto load_g = [&](const uint16_t *of, int col) {  // the lane's row of G (kPoly), ahead of its use
                const int row = row0 + lane, ldg = p.ldg[w.cls];
                const uint4 *from = reinterpret_cast<const uint4 *>(of + w.z * p.g_batch[w.cls] + static_cast<int64_t>(row) * ldg + col);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    g[k] = make_uint4(0u, 0u, 0u, 0u);
                    if (row < rows && col + 8 * k < ldg) g[k] = __ldg(from + k);
                }
            };
            if constexpr (EPI == kPoly) load_g(p.g[w.cls], w.n0 + kWarpCols * half);
            if (!wait_or_abort(sm, &sm.tfull[buf], (local >> 1) & 1u, p.wait_ns, p.status, lane)) break;
            tc_fence_after_sync();
            const uint32_t acc = tmem + (static_cast<uint32_t>(32 * q) << 16) + static_cast<uint32_t>(BN * buf + kWarpCols * half);
#pragma unroll 1
            for (int i = 0; i < kWarpCols / 32; ++i) {
                uint32_t r[32];
                tmem_ld_32x32b_x32(acc + 32 * i, r);
                tmem_ld_wait();
                if (i == kWarpCols / 32 - 1) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster_cta_scope(tempty0 + 8u * buf);
                }
                const int col = w.n0 + kWarpCols * half + 32 * i;
                if (row0 >= rows || col >= cols) continue;
                float v[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = alpha * __uint_as_float(r[k]);
                if constexpr (EPI == kPoly) {
                    auto add_g = [&] {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t xs[4] = {g[k].x, g[k].y, g[k].z, g[k].w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&xs[j]));
                                v[8 * k + 2 * j] = fmaf(p.beta, f.x, v[8 * k + 2 * j]);
                                v[8 * k + 2 * j + 1] = fmaf(p.beta, f.y, v[8 * k + 2 * j + 1]);
                            }
                        }
                    };
                    add_g();
                    if (p.g_lo[w.cls]) {
                        load_g(p.g_lo[w.cls], col);
                        add_g();
                    }
                    if (i + 1 < kWarpCols / 32) load_g(p.g[w.cls], col + 32);
                    if (col <= row0 + 31 && row0 <= col + 31) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (row0 + lane == col + k) v[k] += p.gamma;
                    }
                }
                if constexpr (EPI == kOut) {
                    values_to_u(stage_buf, out, p.first[w.cls] + w.z, v, row0, col, rows, cols, lane);
                } else {
                    uint32_t h[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) h[k] = half2_bits(v[2 * k], v[2 * k + 1]);
                    store(&maps.d, h, false, col, row0, w.z);
                    if (w.mirror) store(&maps.d, h, true, row0, col, w.z);
                    if (p.store_lo[w.cls]) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[k]));
                            h[k] = half2_bits(v[2 * k] - f.x, v[2 * k + 1] - f.y);
                        }
                        store(&maps.d_lo, h, false, col, row0, w.z);
                        if (w.mirror) store(&maps.d_lo, h, true, row0, col, w.z);
                    }
                }
            }
        }
        if (e) bulk_wait_group0();
        __syncwarp();
    }
    // the pair's MMAs are complete and read, and no arrival targets a CTA that has left
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc_pair(tmem, kTmemCols);
}

// ------------------------------------- all products of a matrix of few rows
// A pair of CTAs takes a matrix of m <= 256 through all steps: the results of m x m
// stay in shared memory, each CTA with h = m / 2 rows (up to a multiple of 32) of all of
// them, and X goes through L2.  CTA r has rows h r .. of A and, the first h of its 128,
// of B, so that a pair MMA of 256 x 2h gives row h r + i in lane i of CTA r; rows h .. 127
// of A are whatever lies there, and so are the accumulators' lanes, which nothing reads.
// G and its powers have zeros in columns m .. 2h.  Every sum is that of the launches, bit
// for bit.  Bound by latency: seven products in a row, each waiting for the one before,
// 1.6 us each (the cluster-wide release and acquire of a square 0.2 of it) where a launch
// takes 2.9: one [48, 80] 70 -> 38 us a call, 24 matrices of [128, 1536] and 11 smaller
// ones 145 -> 105.
//   warp 0       TMA producer (both CTAs): X's rows for G, its columns for B X
//   warp 1       MMA issuer (even CTA); tensor memory
//   warps 4..11  epilogue (both CTAs): warp 4 + 4h + q has rows 32q .. and every second
//                32 columns
struct SmallClass {
    CUtensorMap rows[2], cols[2], lo, block[2];  // X and the next X: 64 x 128, 64 x 64 (and its lo), 32 x 32
    int m, n, first;    // first: of the class's matrices
    int passes;         // of X X^T: 3 with hi and lo, 1
    bool precise;       // all results are hi and lo: lo is the second block of a square
};
struct StepPair {
    bool pair, glo, last;  // glo: G's lost digits are kept for T
    float g, c0, b0, a0, t, g1, c1, b1, a1, p, x;
};
struct SmallLo {  // the same of all lo's
    CUtensorMap rows[2], next_cols, block[2];
};
struct NoLo {};
template <bool PRECISE>  // some classes are (launches copy their parameters)
struct MuonSmall {
    int classes, units, steps;
    bool lo;  // the first X has digits in its lo
    int unit0[kMaxClasses + 1];
    SmallClass cls[kMaxClasses];
    std::conditional_t<PRECISE, SmallLo, NoLo> lo_of[kMaxClasses];
    StepPair step[kMaxSteps / 2 + 1];
    const MuonScale *scale;
    int32_t *status;
    uint64_t wait_ns;
};
constexpr int kSmallStages = 8, kSquareBytes = 4 * kBM * 128;
struct SmallSmem {
    // 0: G, G1, B1 B0 (or the last B0).  1: G's lo, T', B1.  2: B0.  Chunks of 64 columns,
    // [128][64] with the 128-byte swizzle.  1 and 2 are the ring of X's k-blocks meanwhile.
    // Up to 32 rows lo lies where the second chunk would.
    alignas(1024) uint8_t square[3][kSquareBytes];
    alignas(1024) uint8_t stage[kEpiWarps][4096];
    uint64_t full[kSmallStages], empty[kSmallStages];
    uint64_t tfull[2], tempty[2];
    uint64_t stored;  // (even CTA's) a result of m x m lies in both CTAs' shared memory
    uint64_t ring;    // 1 and 2 have been read
    uint64_t next;    // this CTA's rows of the next X are in memory
    uint64_t drain;
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(2 * kSquareBytes == kSmallStages * kBM * 128, "the ring is two squares");
struct SmallUnit {
    int cls, z, h, kb_m, kb_n, tiles;
};
// Over P and X: 2, X's lo after its hi; 3, then P's lo with X's hi.
PURO_DEV int x_passes(bool lo, bool precise, int s) { return precise ? 3 : s == 0 && lo ? 2 : 1; }
template <bool PRECISE>
PURO_DEV SmallUnit small_unit(const MuonSmall<PRECISE> &p, int u) {
    SmallUnit w;
    w.cls = 0;
    while (w.cls + 1 < p.classes && u >= p.unit0[w.cls + 1]) ++w.cls;
    const int m = p.cls[w.cls].m, n = p.cls[w.cls].n;
    w.z = u - p.unit0[w.cls];
    w.h = (m + 63) / 64 * 32;
    w.kb_m = (m + kBK - 1) / kBK;
    w.kb_n = (n + kBK - 1) / kBK;
    w.tiles = (n + 255) / 256;
    return w;
}

template <bool PRECISE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    muon_small_kernel(const __grid_constant__ MuonSmall<PRECISE> p, const __grid_constant__ MuonOut out) {
    constexpr uint32_t kBlockBytes = kBM * 128;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    SmallSmem &sm = *reinterpret_cast<SmallSmem *>(smem_raw);
    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = __shfl_sync(0xFFFFFFFFu, static_cast<int>(cluster_ctarank()), 0);
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kSmallStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.tfull[b], 1);
            mbar_init(&sm.tempty[b], 2 * kEpiWarps);
        }
        mbar_init(&sm.stored, 2 * kEpiWarps);
        mbar_init(&sm.ring, kEpiWarps);
        mbar_init(&sm.next, kEpiWarps);
        mbar_init(&sm.drain, 1);
        sm.abort_flag = 0;
        fence_mbarrier_init();
    }
    __syncthreads();
    if (warp == 1) {
        tmem_alloc_pair(&sm.tmem_base, kTmemCols);
        tmem_relinquish_alloc_permit_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    cluster_arrive();
    cluster_wait();  // both CTAs' barriers exist
    const uint32_t tmem = sm.tmem_base;
    uint8_t *const ring = sm.square[1];

    if (warp == 0) {
        // ------------------------------------------------ TMA producer
        const uint32_t e = elect_one();
        const uint32_t full0 = mapa_shared(smem_u32(&sm.full[0]), 0);
        uint32_t stage = 0, phase = 0, issued = 0, ring_phase = 0, next_phase = 0;
        bool ok = true;
        pdl_wait();
        pdl_launch_dependents();
        auto slot = [&] {  // a free place, or null
            ok = wait_or_abort(sm, &sm.empty[stage], phase ^ 1u, p.wait_ns, p.status, lane);
            if (ok && rank == 0 && e) mbar_arrive_expect_tx(&sm.full[stage], 2u * kBlockBytes);
            return ring + kBlockBytes * stage;
        };
        auto filled = [&] {
            ++issued;
            if (++stage == kSmallStages) {
                stage = 0;
                phase ^= 1u;
            }
        };
        for (int u = pair; u < p.units && ok; u += pairs) {
            const SmallUnit w = small_unit(p, u);
            const SmallClass &c = p.cls[w.cls];
            const bool precise = PRECISE && c.precise;
            for (int s = 0; s < p.steps && ok; ++s) {
                if (s > 0) {
                    ok = wait_or_abort(sm, &sm.next, next_phase, p.wait_ns, p.status, lane);
                    next_phase ^= 1u;
                    fence_proxy_async_global();
                }
                for (int pass = 0; pass < (precise ? c.passes : 1); ++pass)  // hi; hi, lo; lo, hi
                    for (int kb = 0; kb < w.kb_n && ok; ++kb)
                        for (int i = 0; i < (pass == 0 ? 1 : 2); ++i) {
                            uint8_t *to = slot();
                            if (!ok) break;
                            const CUtensorMap *map = &c.rows[s & 1];
                            if constexpr (PRECISE)
                                if (pass + i == 2) map = &p.lo_of[w.cls].rows[s & 1];
                            tma_load_3d_pair_e(e, to, map, full0 + 8u * stage, kb * kBK, w.h * rank, w.z);
                            filled();
                        }
                if (!ok) break;
                ok = wait_or_abort(sm, &sm.ring, ring_phase, p.wait_ns, p.status, lane);
                ring_phase ^= 1u;
                fence_proxy_async_global();
                for (int t = 0; t < w.tiles && ok; ++t)
                    for (int kb = 0; kb < w.kb_m * x_passes(p.lo, precise, s); ++kb) {
                        const CUtensorMap *map = kb / w.kb_m == 1 ? &c.lo : &c.cols[s & 1];
                        if constexpr (PRECISE)
                            if (kb / w.kb_m == 1 && (s & 1)) map = &p.lo_of[w.cls].next_cols;
                        uint8_t *to = slot();
                        if (!ok) break;
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            tma_load_3d_pair_e(e, to + 8192 * i, map, full0 + 8u * stage, 256 * t + 128 * rank + 64 * i,
                                               kb % w.kb_m * kBK, w.z);
                        filled();
                    }
            }
        }
        if (rank == 0) {  // every fill of the ring (both CTAs' copies) lands before the pair exits
            for (uint32_t s = 0; s < kSmallStages; ++s) {
                const uint32_t fills = issued / kSmallStages + (s < issued % kSmallStages ? 1u : 0u);
                if (fills > 0) mbar_wait_bounded(&sm.full[s], (fills - 1u) & 1u, kDrainNs);
            }
        }
        if (!ok) {  // this CTA's copies count on the even CTA's barriers: give those in flight time to land
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < kSettleNs) {
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------ MMA issuer
        const uint32_t e = elect_one();
        uint32_t stage = 0, phase = 0, stored_phase = 0;
        int local = 0;
        bool ok = true;
        // kind::f16, FP32 accumulators, FP16 operands, M = 256
        constexpr uint32_t kIdesc = (1u << 4) | ((256u >> 4) << 24), kXIdesc = kIdesc | (1u << 16) | ((256u >> 3) << 17);
        auto free_buffer = [&] { ok = ok && wait_or_abort(sm, &sm.tempty[local & 1], ((local >> 1) & 1u) ^ 1u, p.wait_ns, p.status, lane); };
        auto done = [&] {
            if (ok) tc_commit_pair_multicast_e(e, &sm.tfull[local & 1], 3);
            ++local;
        };
        auto next_block = [&] {  // of the ring
            ok = ok && wait_or_abort(sm, &sm.full[stage], phase, p.wait_ns, p.status, lane);
            tc_fence_after_sync();
            const uint32_t at = smem_u32(ring + kBlockBytes * stage);
            if (++stage == kSmallStages) {
                stage = 0;
                phase ^= 1u;
            }
            return at;
        };
        auto release = [&](uint32_t at) {
            if (ok) tc_commit_pair_multicast_e(e, &sm.empty[(at - smem_u32(ring)) / kBlockBytes], 3);
        };
        auto wait_stored = [&] {
            ok = ok && wait_or_abort(sm, &sm.stored, stored_phase, p.wait_ns, p.status, lane);
            if (ok) mbar_test_wait_cluster(&sm.stored, stored_phase);  // (complete: acquires what the other CTA's warps released)
            stored_phase ^= 1u;
            tc_fence_after_sync();
        };
        for (int u = pair; u < p.units && ok; u += pairs) {
            const SmallUnit w = small_unit(p, u);
            const SmallClass &c = p.cls[w.cls];
            const bool precise = PRECISE && c.precise;
            const uint32_t idesc = kIdesc | (static_cast<uint32_t>(2 * w.h >> 3) << 17);
            auto square = [&](uint32_t from, uint32_t to, bool more) {  // d (+)= a b^T
                const uint32_t d = tmem + 256u * (local & 1);
                for (int kb = 0; kb < w.kb_m && ok; ++kb)
#pragma unroll
                    for (int k = 0; k < kBK / 16; ++k)
                        mma_pair_f16_e(e, d, smem_desc_k_sw128(from + kBlockBytes * kb + 32 * k), smem_desc_k_sw128(to + kBlockBytes * kb + 32 * k),
                                       idesc, more || kb > 0 || k > 0 ? 1u : 0u);
            };
            for (int s = 0; s < p.steps && ok; ++s) {
                const StepPair &q = p.step[s];
                free_buffer();
                if (local == 0) pdl_wait();  // (the kernel before is not what a bounded wait is for)
                const uint32_t d = tmem + 256u * (local & 1);
                for (int pass = 0; pass < (precise ? c.passes : 1); ++pass)
                    for (int kb = 0; kb < w.kb_n && ok; ++kb) {
                        const uint32_t x = next_block(), y = pass == 0 ? x : next_block();
                        if (!ok) break;
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)
                            mma_pair_f16_e(e, d, smem_desc_k_sw128(x + 32 * k), smem_desc_k_sw128(y + 32 * k), idesc,
                                           pass > 0 || kb > 0 || k > 0 ? 1u : 0u);
                        release(x);
                        if (pass > 0) release(y);
                    }
                done();
                // B0; T' = B0 G; G1 = B0 T; B1; B1 B0
#pragma unroll 1
                for (int i = 1; i < (q.pair ? 6 : 2); ++i) {
                    wait_stored();
                    free_buffer();
                    const uint32_t a = smem_u32(sm.square[i == 2 || i == 3 ? 2 : i == 5 ? 1 : 0]);
                    const uint32_t b = smem_u32(sm.square[i == 3 ? 1 : i == 5 ? 2 : 0]), g_lo = smem_u32(sm.square[1]);
                    for (int pass = 0; pass < (precise ? 3 : i == 2 && q.glo ? 2 : 1); ++pass)
                        square(pass == 2 ? a + kBlockBytes : a, pass != 1 ? b : precise ? b + kBlockBytes : g_lo, pass > 0);
                    done();
                }
                wait_stored();
                for (int t = 0; t < w.tiles && ok; ++t) {
                    free_buffer();
                    const uint32_t dx = tmem + 256u * (local & 1), a = smem_u32(sm.square[0]);
                    for (int kb = 0; kb < w.kb_m * x_passes(p.lo, precise, s); ++kb) {
                        const uint32_t x = next_block();
                        if (!ok) break;
                        const uint32_t from = kb / w.kb_m == 2 ? a + kBlockBytes : a + kBlockBytes * (kb % w.kb_m);
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)
                            mma_pair_f16_e(e, dx, smem_desc_k_sw128(from + 32 * k), smem_desc_mn_sw128(x + 2048 * k, 8192), kXIdesc,
                                           kb > 0 || k > 0 ? 1u : 0u);
                        release(x);
                    }
                    done();
                }
            }
        }
        if (e) {  // all MMAs issued are complete before teardown
            tc_commit_pair(&sm.drain);
            mbar_wait_bounded(&sm.drain, 0, kDrainNs);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) >> 2;
        const uint32_t e = elect_one();
        uint8_t *stage_buf = sm.stage[warp - 4];
        const uint32_t tempty0 = mapa_shared(smem_u32(&sm.tempty[0]), 0), stored0 = mapa_shared(smem_u32(&sm.stored), 0);
        const uint32_t own_ring = mapa_shared(smem_u32(&sm.ring), rank), own_next = mapa_shared(smem_u32(&sm.next), rank);
        uint32_t pieces = 0;
        int local = 0;
        bool ok = true;
        // one 32 x 32 block by way of the next half of the staging tile
        auto store = [&](const CUtensorMap *map, const uint32_t(&x)[16], int col, int row, int z) {
            uint8_t *to = stage_buf + 2048 * (pieces & 1u);
            if (e) bulk_wait_group_read<1>();
            __syncwarp();
            stage_rows(to, x, lane);
            fence_proxy_async_smem();
            __syncwarp();
            tma_store_3d_e(e, map, to, col, row, z);
            ++pieces;
        };
        pdl_wait();
        for (int u = pair; u < p.units && ok; u += pairs) {
            const SmallUnit w = small_unit(p, u);
            const SmallClass &c = p.cls[w.cls];
            const bool precise = PRECISE && c.precise;
            const int row0 = w.h * rank + 32 * q, row = 32 * q + lane;  // of X, of the CTA's
            const bool some = 32 * q < w.h;
            auto wait_acc = [&] {
                ok = wait_or_abort(sm, &sm.tfull[local & 1], (local >> 1) & 1u, p.wait_ns, p.status, lane);
                tc_fence_after_sync();
                return tmem + (static_cast<uint32_t>(32 * q) << 16) + 256u * (local & 1);
            };
            auto read_acc = [&] {  // the accumulator is free
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_cta_scope(tempty0 + 8u * (local & 1));
                ++local;
            };
            auto arrive_own = [&](uint32_t bar) {
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster_cta_scope(bar);
            };
            // pieces of 8 values of 32 columns from col on
            auto piece = [&](int at, int block, int col, int k) {
                return reinterpret_cast<uint4 *>(sm.square[at] + kBlockBytes * (block + (col >> 6)) + 128 * row +
                                                 16 * ((((col & 63) >> 3) + k) ^ (row & 7)));
            };
            // alpha D, or alpha D + beta G + gamma I, of m x m, to square `to`; the digits that it loses to `lo`
            auto square = [&](int to, int lo, float alpha, bool poly, float beta, float gamma) {
                const uint32_t acc = wait_acc();
                if (!ok) return;
                for (int col = 32 * half; some && col < 2 * w.h; col += 64) {
                    uint32_t r[32];
                    tmem_ld_32x32b_x32(acc + col, r);
                    tmem_ld_wait();
                    float v[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = alpha * __uint_as_float(r[k]);
                    if (poly) {
#pragma unroll 1
                        for (int block = 0; block < (precise ? 2 : 1); ++block)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint4 g = *piece(0, block, col, k);
                                const uint32_t xs[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&xs[j]));
                                    v[8 * k + 2 * j] = fmaf(beta, f.x, v[8 * k + 2 * j]);
                                    v[8 * k + 2 * j + 1] = fmaf(beta, f.y, v[8 * k + 2 * j + 1]);
                                }
                            }
                        if (col == row0) {
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (lane == k) v[k] += gamma;
                        }
                    }
                    if (col + 32 > c.m) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (col + k >= c.m) v[k] = 0.0f;
                    }
                    uint32_t x[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = half2_bits(v[2 * k], v[2 * k + 1]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) *piece(to, 0, col, k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    if (lo >= 0) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x[k]));
                            x[k] = half2_bits(v[2 * k] - f.x, v[2 * k + 1] - f.y);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) *piece(lo, precise ? 1 : 0, col, k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    }
                }
                read_acc();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(stored0);
            };
            const float r = __ldg(&p.scale[c.first + w.z].r);  // of the first X
            for (int s = 0; s < p.steps && ok; ++s) {
                const StepPair &f = p.step[s];
                // (one piece of code for them all: a call is over before six were fetched)
#pragma unroll 1
                for (int i = 0; i < (f.pair ? 6 : 2) && ok; ++i) {
                    const bool poly = i == 1 || i == 4;
                    const float alpha = i == 0 ? (s == 0 ? f.g * (r * r) : f.g) : i == 1 ? f.c0 : i == 2 ? f.t : i == 3 ? f.g1 : i == 4 ? f.c1 : f.p;
                    const int to = i == 1 && f.pair ? 2 : i == 2 || i == 4 ? 1 : 0;
                    square(to, precise ? to : i == 0 && f.glo ? 1 : -1, alpha, poly, i == 1 ? f.b0 : f.b1, i == 1 ? f.a0 : f.a1);
                }
                if (!ok) break;
                arrive_own(own_ring);  // the last product of squares was complete
                const float alpha = s == 0 ? f.x * r : f.x;
                for (int t = 0; t < w.tiles; ++t) {
                    const uint32_t acc = wait_acc();
                    if (!ok) break;
                    for (int i = half; some && row0 < c.m && i < 8; i += 2) {
                        const int col = 256 * t + 32 * i;
                        if (col >= c.n) break;
                        uint32_t d[32];
                        tmem_ld_32x32b_x32(acc + 32 * i, d);
                        tmem_ld_wait();
                        float v[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = alpha * __uint_as_float(d[k]);
                        if (f.last) {
                            values_to_u(stage_buf, out, c.first + w.z, v, row0, col, c.m, c.n, lane);
                        } else {
                            uint32_t x[16];
#pragma unroll
                            for (int k = 0; k < 16; ++k) x[k] = half2_bits(v[2 * k], v[2 * k + 1]);
                            store(&c.block[(s + 1) & 1], x, col, row0, w.z);
                            if constexpr (PRECISE) {
                                if (precise) {
#pragma unroll
                                    for (int k = 0; k < 16; ++k) {
                                        const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&x[k]));
                                        x[k] = half2_bits(v[2 * k] - y.x, v[2 * k + 1] - y.y);
                                    }
                                    store(&p.lo_of[w.cls].block[(s + 1) & 1], x, col, row0, w.z);
                                }
                            }
                        }
                    }
                    read_acc();
                }
                if (!ok || f.last) break;
                if (e) bulk_wait_group0();
                fence_proxy_async_global();
                arrive_own(own_next);
            }
        }
        if (e) bulk_wait_group0();
        __syncwarp();
    }
    // the pair's MMAs are complete and read, and no arrival targets a CTA that has left
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc_pair(tmem, kTmemCols);
}

// ------------------------------------------------------------------- host
constexpr int64_t kAlign = 256;

// Square ones; X, its lo, the next X; the others' lo where a class keeps all (is_precise).
enum Buffer { kG, kB0, kT, kB1, kX, kXlo, kXnext, kXnextLo, kGlo, kB0lo, kTlo, kB1lo, kBuffers, kNone = -1 };
bool is_square(int b) { return b < kX || b >= kGlo; }
int lo_of(int b) { return b == kX ? kXlo : b == kXnext ? kXnextLo : b + kGlo; }

// Scratch of a chunk.
struct Scratch {
    int64_t bytes = 0;
    int64_t buffer[kBuffers][kMaxClasses];  // offsets; -1: none
    int64_t partial = 0, guess = 0, scale = 0;
};
int64_t tiles_in(int64_t rows, int64_t cols) {
    return (rows + kInRows - 1) / kInRows * ((cols + kInCols - 1) / kInCols);
}
Scratch scratch_of(const puro_muon_matrix_t *mats, const Chunk &c) {
    Scratch s;
    auto take = [&](int64_t bytes) {
        const int64_t at = s.bytes;
        s.bytes += align_up(bytes, kAlign);
        return at;
    };
    int64_t tiles = 0;
    for (int i = 0; i < c.count; ++i) tiles += tiles_in(mats[c.mats[i]].rows, mats[c.mats[i]].cols);
    s.partial = take(8 * tiles);
    s.guess = take(4 * c.count);
    s.scale = take(static_cast<int64_t>(sizeof(MuonScale)) * c.count);
    for (int k = 0; k < c.classes; ++k) {
        const int64_t n = c.first[k + 1] - c.first[k];
        for (int b = 0; b < kBuffers; ++b) {
            const bool there = b <= kXnext || is_precise(c.shape[k].m);
            s.buffer[b][k] = there ? take(n * c.shape[k].m * align_up(is_square(b) ? c.shape[k].m : c.shape[k].n, 8) * 2) : -1;
        }
    }
    return s;
}

// One step's polynomial p(t) = a + b t + c t^2 of the squared singular values, and
// what it does to singular values up to `most`: the bound of |p| and of sigma |p|.
struct Step {
    double a, b, c, most_p, most_out;
};
bool plan_step(const double *abc, double most, Step *s) {
    s->a = abc[0];
    s->b = abc[1];
    s->c = abc[2];
    if (!std::isfinite(s->a) || !std::isfinite(s->b) || !std::isfinite(s->c)) return false;
    const double t1 = most * most;
    auto p = [&](double t) { return s->a + t * (s->b + t * s->c); };
    auto f = [&](double t) { return std::sqrt(t) * std::fabs(p(t)); };
    s->most_p = std::max(std::fabs(s->a), std::fabs(p(t1)));
    s->most_out = f(t1);
    const double v = -s->b / (2 * s->c);  // (c = 0: not finite, no vertex)
    if (v > 0 && v < t1) s->most_p = std::max(s->most_p, std::fabs(p(v)));
    // extremes of sigma p(sigma^2): a + 3 b t + 5 c t^2 = 0
    const double disc = 9 * s->b * s->b - 20 * s->a * s->c;
    auto at = [&](double t) {
        if (t > 0 && t < t1) s->most_out = std::max(s->most_out, f(t));
    };
    if (s->c != 0) {
        if (disc >= 0) {
            at((-3 * s->b + std::sqrt(disc)) / (10 * s->c));
            at((-3 * s->b - std::sqrt(disc)) / (10 * s->c));
        }
    } else if (s->b != 0) {
        at(-s->a / (3 * s->b));
    }
    return s->most_p < 1024 && s->most_out < 1024;
}
constexpr double kMargin = 1.0 + 1.0 / 64;  // of a bound, for what roundings add
// The power of two that puts values up to `most` within FP16, with half of it to spare.
double pow2_for(double most) { return std::ldexp(1.0, most > 0 ? std::min(100, std::ilogb(32768.0 / (most * kMargin))) : 14); }

// (once per device: it costs as much of the host's time as an eighth of a launch)
template <int BN, bool X_MAJOR, int EPI>
cudaError_t product_attribute() {
    static std::atomic<bool> done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_relaxed))) return e;
    e = cudaFuncSetAttribute(muon_product_kernel<BN, X_MAJOR, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(sizeof(ProductSmem<BN>)));
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_relaxed);
    return e;
}
template <bool PRECISE>
cudaError_t small_attribute() {
    static std::atomic<bool> done[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_relaxed))) return e;
    e = cudaFuncSetAttribute(muon_small_kernel<PRECISE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(sizeof(SmallSmem)));
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_relaxed);
    return e;
}
// Pairs of SMs that run pairs of CTAs.
cudaError_t resident_pairs(int *pairs) {
    static int cache[64] = {0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && cache[dev] > 0) {
        *pairs = cache[dev];
        return cudaSuccess;
    }
    e = product_attribute<256, false, kStore>();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    const int sms = sm_count_here();
    cfg.gridDim = dim3(static_cast<unsigned>(sms / 2 * 2), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = sizeof(ProductSmem<256>);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, muon_product_kernel<256, false, kStore>, &cfg) != cudaSuccess || n <= 0) {
        (void)cudaGetLastError();
        n = sms / 2;
    }
    if (dev >= 0 && dev < 64) cache[dev] = n;
    *pairs = n;
    return cudaSuccess;
}

template <int BN, bool X_MAJOR, int EPI>
cudaError_t launch_product(const MuonPhase &p, const OutOf<EPI> &out, int pairs, cudaStream_t s) {
    const cudaError_t e = product_attribute<BN, X_MAJOR, EPI>();
    if (e != cudaSuccess) return e;
    return launch_pdl(muon_product_kernel<BN, X_MAJOR, EPI>, dim3(2 * std::min(p.units, pairs)), dim3(kThreads),
                      sizeof(ProductSmem<BN>), s, p, out);
}

// The products of a chunk, phase after phase.
struct Products {
    const Chunk &c;
    const Scratch &at;
    uint8_t *ws;
    int32_t *status;
    cudaStream_t s;
    int pairs;  // of SMs
    bool small;  // muon_small_kernel takes all of them
    MuonOut out;
    Tiles tiles[kForms];
    // of each buffer: 64 x 128 (A; B of 256 columns), 64 x 64 (B of 128; X), 32 x 32 (D)
    CUtensorMap rows128[kMaxClasses][kBuffers], rows64[kMaxClasses][kBuffers], block[kMaxClasses][kBuffers];

    int64_t ld(int k, bool square) const { return align_up(square ? c.shape[k].m : c.shape[k].n, 8); }
    uint16_t *buffer(int b, int k) const { return reinterpret_cast<uint16_t *>(ws + at.buffer[b][k]); }
    bool precise(int k) const { return is_precise(c.shape[k].m); }

    cudaError_t prepare() {
        for (int form = 0; form < kForms && !small; ++form) {
            Tiles narrow;
            const double narrow_most = deal(c, pairs, &narrow, form, 128), wide_most = deal(c, pairs, &tiles[form], form, 256);
            if (narrow_most < wide_most) tiles[form] = narrow;
            if (!std::isfinite(std::min(narrow_most, wide_most))) return cudaErrorInvalidConfiguration;
        }
        for (int k = 0; k < c.classes; ++k)
            for (int b = 0; b < kBuffers; ++b) {
                if (at.buffer[b][k] < 0 || (small && is_square(b))) continue;
                const bool square = is_square(b);
                const int64_t cols = square ? c.shape[k].m : c.shape[k].n, row = 2 * ld(k, square);
                auto map = [&](CUtensorMap *m, int bx, int by, CUtensorMapSwizzle sw) {
                    return make_batched_map(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, buffer(b, k), cols, c.shape[k].m,
                                            c.first[k + 1] - c.first[k], row, row * c.shape[k].m, bx, by, sw);
                };
                if (!map(&rows128[k][b], 64, 128, CU_TENSOR_MAP_SWIZZLE_128B) || !map(&rows64[k][b], 64, 64, CU_TENSOR_MAP_SWIZZLE_128B) ||
                    !map(&block[k][b], 32, 32, CU_TENSOR_MAP_SWIZZLE_64B))
                    return cudaErrorInvalidValue;
            }
        return cudaSuccess;
    }

    // All products, where small.
    template <bool PRECISE>
    cudaError_t run_small(const StepPair *step, int n, bool lo, const MuonScale *scale) const {
        const cudaError_t e = small_attribute<PRECISE>();
        if (e != cudaSuccess) return e;
        MuonSmall<PRECISE> p{};
        for (int k = 0; k < c.classes; ++k) {
            SmallClass &to = p.cls[p.classes];
            for (int i = 0; i < 2; ++i) {
                const int x = i == 0 ? kX : kXnext;
                to.rows[i] = rows128[k][x];
                to.cols[i] = rows64[k][x];
                to.block[i] = block[k][x];
                if constexpr (PRECISE) {
                    if (!precise(k)) continue;
                    SmallLo &more = p.lo_of[p.classes];
                    more.rows[i] = rows128[k][lo_of(x)];
                    more.block[i] = block[k][lo_of(x)];
                    if (i == 1) more.next_cols = rows64[k][lo_of(x)];
                }
            }
            to.lo = rows64[k][kXlo];
            to.precise = precise(k);
            to.passes = to.precise && c.shape[k].n <= kPreciseGram ? 3 : 1;
            to.m = static_cast<int>(c.shape[k].m);
            to.n = static_cast<int>(c.shape[k].n);
            to.first = c.first[k];
            p.units += c.first[k + 1] - c.first[k];
            p.unit0[++p.classes] = p.units;
        }
        std::copy(step, step + n, p.step);
        p.steps = n;
        p.lo = lo;
        p.scale = scale;
        p.status = status;
        p.wait_ns = wait_timeout_ns();
        return launch_pdl(muon_small_kernel<PRECISE>, dim3(2 * std::min(p.units, pairs)), dim3(kThreads), sizeof(SmallSmem), s, p, out);
    }

    // D = A B^T or (kTimesX) A X, of buffers.
    struct Product {
        Form form;
        int a, b;
        bool b_lo;  // B's lo is added (a second pass over A); a precise class has all products of hi and lo but lo's with lo
        int d;
        bool d_lo;  // the digits that D loses are kept as well; in a precise class they all are
        const MuonScale *scale = nullptr;  // of the first X
        float alpha = 0, beta = 0, gamma = 0;
    };
    template <int EPI, bool X_MAJOR>
    cudaError_t run(const Product &q) const {
        MuonPhase p;
        static_cast<Tiles &>(p) = tiles[q.form];
        for (int k = 0; k < c.classes; ++k) {
            const CUtensorMap *b = X_MAJOR || p.bn == 128 ? rows64[k] : rows128[k];
            const bool all = precise(k);
            // elsewhere G's lo is in B1's place, and read before that is written
            auto lo = [&](int buf) { return !all && buf == kG ? static_cast<int>(kB1) : lo_of(buf); };
            p.passes[k] = all ? (q.form == kGram && c.shape[k].n > kPreciseGram ? 1 : 3) : q.b_lo ? 2 : 1;
            p.store_lo[k] = (all || q.d_lo) && q.d != kNone;
            p.maps[k].a = rows128[k][q.a];
            p.maps[k].b = b[q.b];
            if (p.passes[k] > 1) p.maps[k].b_lo = b[lo(q.b)];
            if (p.passes[k] > 2) p.maps[k].a_lo = rows128[k][lo(q.a)];
            if (q.d != kNone) p.maps[k].d = block[k][q.d];
            if (p.store_lo[k]) p.maps[k].d_lo = block[k][lo(q.d)];
            p.g[k] = buffer(kG, k);
            p.g_lo[k] = all ? buffer(kGlo, k) : nullptr;
            p.ldg[k] = static_cast<int>(ld(k, true));
            p.g_batch[k] = c.shape[k].m * ld(k, true);
        }
        p.alpha = q.alpha;
        p.beta = q.beta;
        p.gamma = q.gamma;
        p.scale = q.scale;
        p.squared = q.form == kGram;
        p.status = status;
        p.wait_ns = wait_timeout_ns();
        // kind::f16, FP32 accumulators, FP16 operands; B N-major for X; N, M = 256 (a pair MMA)
        p.idesc = (1u << 4) | (X_MAJOR ? 1u << 16 : 0u) | (static_cast<uint32_t>(p.bn >> 3) << 17) | ((256u >> 4) << 24);
        OutOf<EPI> to{};
        if constexpr (EPI == kOut) to = out;
        return p.bn == 256 ? launch_product<256, X_MAJOR, EPI>(p, to, pairs, s) : launch_product<128, X_MAJOR, EPI>(p, to, pairs, s);
    }
};

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

puro_status_t check_matrix(const puro_muon_matrix_t &a) {
    if (a.rows < 0 || a.cols < 0 || a.reserved != 0) return PURO_ERR_INVALID_ARG;
    if ((a.grad_type != PURO_BF16 && a.grad_type != PURO_F32) || (a.u_type != PURO_BF16 && a.u_type != PURO_F32))
        return PURO_ERR_INVALID_ARG;
    if (empty(a)) return PURO_OK;
    if (!a.grad || !a.u || !aligned(a.grad, a.grad_type == PURO_F32 ? 4 : 2) || !aligned(a.u, a.u_type == PURO_F32 ? 4 : 2) ||
        !aligned(a.momentum, 4))
        return PURO_ERR_INVALID_ARG;
    if (a.grad_stride < 0 || (a.rows > 1 && a.u_stride < a.cols)) return PURO_ERR_INVALID_ARG;
    if (a.rows > (1 << 20) || a.cols > (1 << 20)) return PURO_ERR_UNSUPPORTED;
    return PURO_OK;
}

cudaError_t run_chunk(const puro_muon_matrix_t *mats, const Chunk &c, double mu, int nesterov, const Step *steps, int n_steps,
                      uint8_t *ws, int32_t *status, cudaStream_t s) {
    const Scratch at = scratch_of(mats, c);
    int pairs = 0;
    cudaError_t e = resident_pairs(&pairs);
    if (e != cudaSuccess) return e;
    Products run{c, at, ws, status, s, pairs};
    run.small = small_pays(c, pairs, n_steps);
    e = run.prepare();
    if (e != cudaSuccess) return e;
    // the update, its norm, X
    MuonIn in{};
    in.count = c.count;
    in.mu = static_cast<float>(mu);
    in.nesterov = nesterov;
    in.store_lo = n_steps > 1;
    for (int k = 0; k < c.classes; ++k) in.store_lo = in.store_lo || is_precise(c.shape[k].m);
    in.partial = reinterpret_cast<double *>(ws + at.partial);
    in.guess = reinterpret_cast<float *>(ws + at.guess);
    in.scale = reinterpret_cast<MuonScale *>(ws + at.scale);
    for (int k = 0; k < c.classes; ++k)
        for (int i = c.first[k]; i < c.first[k + 1]; ++i) {
            const puro_muon_matrix_t &a = mats[c.mats[i]];
            const int64_t z = (i - c.first[k]) * c.shape[k].m * run.ld(k, false);
            MatIn &to = in.mat[i];
            to.grad = a.grad;
            to.momentum = a.momentum;
            to.stride = a.rows > 1 ? a.grad_stride : a.cols;
            to.rows = static_cast<int>(a.rows);
            to.cols = static_cast<int>(a.cols);
            to.ldx = static_cast<int>(run.ld(k, false));
            to.hi = run.buffer(kX, k) + z;
            to.lo = run.buffer(kXlo, k) + z;
            const bool tall = a.rows > a.cols, bf16 = a.grad_type == PURO_BF16, f32 = a.u_type == PURO_F32;
            const int64_t us = a.rows > 1 ? a.u_stride : a.cols;
            to.flags = (bf16 ? kGradBf16 : 0) | (tall ? kTall : 0);
            if (a.cols % 4 == 0 && aligned(a.momentum, 16)) {
                to.flags |= kVectors;
                if (aligned(a.grad, bf16 ? 8 : 16) && to.stride % 4 == 0) to.flags |= kGradVectors;
            }
            run.out.u[i] = a.u;
            run.out.stride[i] = us;
            run.out.flags[i] = (tall ? kTall : 0) | (f32 ? kOutF32 : 0);
            if (a.cols % (f32 ? 4 : 8) == 0 && us % (f32 ? 4 : 8) == 0 && aligned(a.u, 16)) run.out.flags[i] |= kOutVectors;
            in.tile0[i + 1] = in.tile0[i] + static_cast<int>(tiles_in(a.rows, a.cols));
        }
    e = launch_pdl(muon_update_kernel, dim3(std::min(in.tile0[c.count], 8 * pairs)), dim3(kInThreads), 0, s, in);
    int widest = 0;  // tiles of a matrix
    for (int i = 0; i < c.count; ++i) widest = std::max(widest, in.tile0[i + 1] - in.tile0[i]);
    // (a block holds an SM from the product behind, whose shared memory does not fit beside)
    const dim3 blocks(std::min((widest + 7) / 8, std::max(1, 2 * pairs / c.count)), c.count);
    if (e == cudaSuccess) e = launch_pdl(muon_norm_kernel, blocks, dim3(kInThreads), 0, s, in);
    // the steps, two at a time: what each product's results are scaled with
    StepPair plan[kMaxSteps / 2 + 1];
    int n_plan = 0;
    double most = 1.0, sx = 1.0;  // (the first X's power of two is in its MuonScale)
    for (int i = 0; i < n_steps;) {
        const bool pair = i + 1 < n_steps;
        const Step &s0 = steps[i];
        StepPair &f = plan[n_plan++];
        const double sg = pow2_for(most * most), sb = pow2_for(s0.most_p);
        f.pair = pair;
        f.glo = pair && i > 0;
        f.g = static_cast<float>(sg / (sx * sx));
        f.c0 = static_cast<float>(s0.c * sb / (sg * sg));
        f.b0 = static_cast<float>(s0.b * sb / sg);
        f.a0 = static_cast<float>(s0.a * sb);
        double sp = sb, bound = s0.most_out * kMargin;
        if (pair) {
            const Step &s1 = steps[i + 1];
            const double st = pow2_for(most * most * s0.most_p), sg1 = pow2_for(bound * bound), sb1 = pow2_for(s1.most_p);
            f.t = static_cast<float>(st / (sg * sb));
            f.g1 = static_cast<float>(sg1 / (st * sb));
            f.c1 = static_cast<float>(s1.c * sb1 / (sg1 * sg1));
            f.b1 = static_cast<float>(s1.b * sb1 / sg1);
            f.a1 = static_cast<float>(s1.a * sb1);
            sp = pow2_for(s0.most_p * s1.most_p);
            f.p = static_cast<float>(sp / (sb1 * sb));
            bound = s1.most_out * kMargin;
        }
        i += pair ? 2 : 1;
        f.last = i == n_steps;
        const double next = f.last ? 1.0 : pow2_for(bound);
        f.x = static_cast<float>(next / (sp * sx));
        sx = next;
        most = bound;
    }
    if (run.small && e == cudaSuccess) {
        bool any = false;
        for (int k = 0; k < c.classes; ++k) any = any || is_precise(c.shape[k].m);
        return any ? run.run_small<true>(plan, n_plan, n_steps > 1, in.scale) : run.run_small<false>(plan, n_plan, n_steps > 1, in.scale);
    }
    for (int i = 0; i < n_plan && e == cudaSuccess; ++i) {
        const StepPair &f = plan[i];
        const MuonScale *scale = i == 0 ? in.scale : nullptr;
        const int x = i & 1 ? kXnext : kX, y = i & 1 ? kX : kXnext;
        const bool lo = i == 0 && n_steps > 1;
        // G = X X^T;  B0 = a I + b G + c G^2
        e = run.run<kStore, false>({kGram, x, x, false, kG, f.glo, scale, f.g});
        if (e == cudaSuccess) e = run.run<kPoly, false>({kSquareSym, kG, kG, false, kB0, false, nullptr, f.c0, f.b0, f.a0});
        int product = kB0;
        if (f.pair) {
            // T^T = B0 G;  G = B0 T;  B1;  T = B1 B0
            if (e == cudaSuccess) e = run.run<kNext, false>({kSquare, kB0, kG, f.glo, kT, false, nullptr, f.t});
            if (e == cudaSuccess) e = run.run<kStore, false>({kSquareSym, kB0, kT, false, kG, false, nullptr, f.g1});
            if (e == cudaSuccess) e = run.run<kPoly, false>({kSquareSym, kG, kG, false, kB1, false, nullptr, f.c1, f.b1, f.a1});
            if (e == cudaSuccess) e = run.run<kNext, false>({kSquare, kB1, kB0, false, kT, false, nullptr, f.p});
            product = kT;
        }
        if (e != cudaSuccess) break;
        if (f.last)
            e = run.run<kOut, true>({kTimesX, product, x, lo, kNone, false, scale, f.x});
        else
            e = run.run<kNext, true>({kTimesX, product, x, lo, y, false, scale, f.x});
    }
    return e;
}

}  // namespace
}  // namespace puro

using namespace puro;

#define PURO_MUON_API extern "C" __attribute__((visibility("default")))

PURO_MUON_API size_t puro_muon_direction_workspace_size(const puro_muon_matrix_t *mats, int32_t count) {
    if (!mats || count <= 0) return 0;
    for (int32_t i = 0; i < count; ++i)
        if (check_matrix(mats[i]) != PURO_OK) return 0;
    int64_t most = 0;
    for (int at = 0; at < count;) {  // the chunks use the scratch one after the other
        Chunk c;
        at = take_chunk(mats, at, count, &c);
        most = std::max(most, scratch_of(mats, c).bytes);
    }
    return static_cast<size_t>(most);
}

PURO_MUON_API puro_status_t puro_muon_direction_grouped(const puro_muon_matrix_t *mats, int32_t count, double momentum,
                                                        int32_t nesterov, const double *coefficients, int32_t steps,
                                                        void *workspace, size_t workspace_bytes, int32_t *dev_status,
                                                        void *stream) {
    if (count < 0 || (count > 0 && !mats)) return PURO_ERR_INVALID_ARG;
    if (!(momentum >= 0.0 && momentum <= 1.0)) return PURO_ERR_INVALID_ARG;
    if (steps < 1 || steps > kMaxSteps || !coefficients || !aligned(dev_status, 4)) return PURO_ERR_INVALID_ARG;
    Step plan[kMaxSteps];
    double most = 1.0;
    for (int i = 0; i < steps; ++i) {
        if (!plan_step(coefficients + 3 * i, most, &plan[i])) return PURO_ERR_INVALID_ARG;
        most = plan[i].most_out * kMargin;
    }
    bool any = false;
    for (int32_t i = 0; i < count; ++i) {
        const puro_status_t st = check_matrix(mats[i]);
        if (st != PURO_OK) return st;
        any = any || !empty(mats[i]);
    }
    if (!any) return PURO_OK;
    {
        const std::unique_ptr<Place[]> places(new (std::nothrow) Place[3 * static_cast<size_t>(count)]);
        if (!places) return PURO_ERR_UNSUPPORTED;
        if (writes_overlap(mats, count, places.get())) return PURO_ERR_INVALID_ARG;
    }
    const size_t need = puro_muon_direction_workspace_size(mats, count);
    if (!workspace || !aligned(workspace, kAlign) || workspace_bytes < need) return PURO_ERR_INVALID_ARG;
    for (int at = 0; at < count;) {
        Chunk c;
        at = take_chunk(mats, at, count, &c);
        if (c.count == 0) break;
        if (run_chunk(mats, c, momentum, nesterov != 0, plan, steps, static_cast<uint8_t *>(workspace), dev_status,
                      static_cast<cudaStream_t>(stream)) != cudaSuccess)
            return PURO_ERR_CUDA;
    }
    return PURO_OK;
}
