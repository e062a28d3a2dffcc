// rotation.cuh -- the position rotation of query and key heads in registers: which
// channels a lane holds, their pairs, and turning the pairs by their angles.  Shared
// by the kernels that normalise heads first (qknorm.cu) and those that do not
// (rope.cu).
//
// A head of D channels belongs to a group of G lanes, 16 channels a lane in two
// 16-byte chunks that hold both channels of each of its pairs, so the rotation
// needs no exchange between lanes.
#pragma once

#include <cuda_bf16.h>

#include "internal.h"
#include "ptx.cuh"
#include "quant_math.cuh"

namespace puro {

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
// A token's row: live, padding (at a negative position), or one that cannot be
// rotated.
enum QkRow : int { kRowLive, kRowPad, kRowOut };

// What a row that is not live counts as: zeros for padding, whatever it holds,
// and NaN past the tables.
PURO_DEV void replace_row(QkRow row, uint4 (&w)[2]) {
    const uint32_t v = row == kRowPad ? 0u : 0x7FC07FC0u;
    w[0] = w[1] = make_uint4(v, v, v, v);
}

inline int group_lanes(int D) { return D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// kern<G, INTER> for the group's lanes and the kind of pairs
#define PURO_QK_KERNEL(kern, p)                                                                      \
    (group_lanes((p).D) == 4   ? ((p).inter ? kern<4, true> : kern<4, false>)                         \
     : group_lanes((p).D) == 8 ? ((p).inter ? kern<8, true> : kern<8, false>)                         \
                               : ((p).inter ? kern<16, true> : kern<16, false>))

}  // namespace puro
