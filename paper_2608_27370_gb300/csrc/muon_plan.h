// muon_plan.h -- who computes what of the Muon directions' products (see muon.cu): the
// matrices of one series of launches, the tiles of a product and the pairs of CTAs
// that take them, and which matrices one kernel takes through all steps.  Host code
// without a CUDA call, and the walk through the tiles, which the kernels share.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "puro_fp8.h"

#ifdef __CUDACC__
#define PURO_PLAN __host__ __device__ __forceinline__
#else
#define PURO_PLAN inline
#endif

namespace puro {

constexpr int kMaxClasses = 8;   // shapes of one launch (their tensor maps are kernel parameters)
constexpr int kMaxMats = 128;    // matrices of one launch
constexpr int kBK = 64;          // of a k-block
constexpr int kMaxSegments = 24;  // 17 for the first of eight shapes, one at least for each of the others
constexpr int kSmallMost = 256;  // rows (or columns) of a matrix that muon_small_kernel takes

// The tiles of a product, and who takes them.
struct Tiles {
    int bn;
    int classes, units;
    int unit0[kMaxClasses + 1];  // first tile of each class
    int per[kMaxClasses];        // tiles of a matrix
    int tiles_n[kMaxClasses], tiles_m[kMaxClasses];
    int rows[kMaxClasses], cols[kMaxClasses];  // of D
    int kb[kMaxClasses];         // k-blocks of B (of lo as many more)
    int first[kMaxClasses];      // the class's first matrix
    int segments;                // of tiles, each dealt to a range of the pairs in turn
    int from[kMaxSegments], to[kMaxSegments];
    int16_t pair0[kMaxSegments], pairs[kMaxSegments];
};
// A pair's units, in order.
struct Walk {
    int segment = 0, u = -1;
    PURO_PLAN int next(const Tiles &p, int pair) {
        for (; segment < p.segments; ++segment, u = -1) {
            if (u < 0) {
                const int i = pair - p.pair0[segment];
                if (i < 0 || i >= p.pairs[segment]) continue;
                u = p.from[segment] + i;
            } else {
                u += p.pairs[segment];
            }
            if (u < p.to[segment]) return u;
        }
        return -1;
    }
};
struct Unit {
    int cls, z, m0, n0, kb;
    bool mirror;  // off the diagonal of a symmetric D: stored transposed as well
};

template <int BN, bool SYM>
PURO_PLAN Unit unit_of(const Tiles &p, int u) {
    Unit w;
    w.cls = 0;
    while (w.cls + 1 < p.classes && u >= p.unit0[w.cls + 1]) ++w.cls;
    int i = u - p.unit0[w.cls];
    w.z = i / p.per[w.cls];
    i -= w.z * p.per[w.cls];
    w.kb = p.kb[w.cls];
    if constexpr (SYM) {
        constexpr int kAcross = 256 / BN;
        const int n = p.tiles_n[w.cls];
        int row = 0;
        while (i >= n - kAcross * row) {
            i -= n - kAcross * row;
            ++row;
        }
        w.m0 = 256 * row;
        w.n0 = BN * (kAcross * row + i);
        w.mirror = w.n0 >= w.m0 + 256;
    } else {  // the rows of B fastest: a wave shares columns of X
        const int tm = p.tiles_m[w.cls];
        w.m0 = 256 * (i % tm);
        w.n0 = BN * (i / tm);
        w.mirror = false;
    }
    return w;
}

inline int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

struct Shape {
    int64_t m, n;
    bool operator==(const Shape &o) const { return m == o.m && n == o.n; }
};
inline Shape shape_of(const puro_muon_matrix_t &a) { return {std::min(a.rows, a.cols), std::max(a.rows, a.cols)}; }
inline bool empty(const puro_muon_matrix_t &a) { return a.rows == 0 || a.cols == 0; }

// The bytes of a matrix: rows that are `pitch` apart.
struct Bytes {
    uintptr_t from;
    int64_t rows, row, pitch;
    uintptr_t end() const { return from + static_cast<uintptr_t>((rows - 1) * pitch + row); }
};
inline Bytes bytes_of(const void *p, int64_t rows, int64_t cols, int64_t stride, int64_t size) {
    const bool one = rows == 1 || stride == 0;  // (a stride of 0: one row, read again)
    stride = std::min(stride, int64_t{1} << 40);  // (more than any memory has)
    return {reinterpret_cast<uintptr_t>(p), one ? 1 : rows, cols * size, one ? cols * size : stride * size};
}
inline bool share(const Bytes &a, const Bytes &b) {
    if (a.from >= b.end() || b.from >= a.end()) return false;
    if (a.pitch == b.pitch && a.row <= a.pitch && b.row <= b.pitch) {  // columns of one wider matrix, say
        const Bytes &x = a.from <= b.from ? a : b, &y = a.from <= b.from ? b : a;
        const int64_t d = static_cast<int64_t>(y.from - x.from), row = d / x.pitch, at = d % x.pitch;
        return (at < x.row && row < x.rows) || (at + y.row > x.pitch && row + 1 < x.rows);
    }
    const Bytes &few = a.rows <= b.rows ? a : b, &many = a.rows <= b.rows ? b : a;
    for (int64_t i = 0; i < few.rows; ++i) {  // the first of `many` that ends behind the row's start
        const uintptr_t start = few.from + static_cast<uintptr_t>(i * few.pitch);
        const int64_t before = start < many.from + static_cast<uintptr_t>(many.row)
                                   ? 0 : static_cast<int64_t>(start - many.from - static_cast<uintptr_t>(many.row)) / many.pitch + 1;
        if (before < many.rows && many.from + static_cast<uintptr_t>(before * many.pitch) < start + static_cast<uintptr_t>(few.row)) return true;
    }
    return false;
}
// Whether something that a call writes lies where something else of it does.  Only a
// matrix's u may lie in its own gradient, which has been read by then.  `at`: 3 count places.
struct Place {
    Bytes bytes;
    int32_t mat;
    enum : int32_t { kGrad, kMomentum, kU } what;
};
inline bool writes_overlap(const puro_muon_matrix_t *mats, int count, Place *at) {
    int n = 0;
    for (int i = 0; i < count; ++i) {
        const puro_muon_matrix_t &a = mats[i];
        if (empty(a)) continue;
        at[n++] = {bytes_of(a.grad, a.rows, a.cols, a.grad_stride, a.grad_type == PURO_F32 ? 4 : 2), i, Place::kGrad};
        if (a.momentum) at[n++] = {bytes_of(a.momentum, a.rows, a.cols, a.cols, 4), i, Place::kMomentum};
        at[n++] = {bytes_of(a.u, a.rows, a.cols, a.u_stride, a.u_type == PURO_F32 ? 4 : 2), i, Place::kU};
    }
    std::sort(at, at + n, [](const Place &x, const Place &y) { return x.bytes.from < y.bytes.from; });
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n && at[j].bytes.from < at[i].bytes.end(); ++j) {
            const Place &x = at[i], &y = at[j];
            if (x.what == Place::kGrad && y.what == Place::kGrad) continue;
            if (x.mat == y.mat && x.what != Place::kMomentum && y.what != Place::kMomentum) continue;
            if (share(x.bytes, y.bytes)) return true;
        }
    return false;
}

template <class Less>
void sort_few(int *v, int n, Less less) {
    for (int i = 1; i < n; ++i)
        for (int j = i; j > 0 && less(v[j], v[j - 1]); --j) std::swap(v[j], v[j - 1]);
}

// The matrices of one series of launches: some in a row of the table, by shape.
struct Chunk {
    int count = 0, classes = 0;
    int mats[kMaxMats];  // their places in the table, class by class
    Shape shape[kMaxClasses];
    int first[kMaxClasses + 1];
};
// Takes matrices from `at` on while they fit one chunk, and returns where it ended.
inline int take_chunk(const puro_muon_matrix_t *mats, int at, int count, Chunk *c) {
    *c = Chunk{};
    int cls[kMaxMats];
    int n[kMaxClasses] = {};
    for (; at < count && c->count < kMaxMats; ++at) {
        if (empty(mats[at])) continue;
        const Shape s = shape_of(mats[at]);
        int k = 0;
        while (k < c->classes && !(c->shape[k] == s)) ++k;
        if (k == kMaxClasses) break;
        if (k == c->classes) c->shape[c->classes++] = s;
        cls[c->count] = k;
        c->mats[c->count++] = at;
        ++n[k];
    }
    // classes of the longest rows first: their tiles are the long ones
    int order[kMaxClasses], place[kMaxClasses];
    for (int k = 0; k < c->classes; ++k) order[k] = k;
    sort_few(order, c->classes, [&](int a, int b) {
        return c->shape[a].n != c->shape[b].n ? c->shape[a].n > c->shape[b].n
                                              : c->shape[a].m != c->shape[b].m ? c->shape[a].m > c->shape[b].m : a < b;
    });
    Shape sorted[kMaxClasses];
    int next[kMaxClasses];
    c->first[0] = 0;
    for (int k = 0; k < c->classes; ++k) {
        place[order[k]] = k;
        sorted[k] = c->shape[order[k]];
        next[k] = c->first[k];
        c->first[k + 1] = c->first[k] + n[order[k]];
    }
    int by[kMaxMats];
    for (int i = 0; i < c->count; ++i) by[next[place[cls[i]]]++] = c->mats[i];
    std::copy(by, by + c->count, c->mats);
    std::copy(sorted, sorted + c->classes, c->shape);
    return at;
}

enum Form { kGram, kSquareSym, kSquare, kTimesX, kForms };  // X X^T; m x m, symmetric or not; m x m times X
// Matrices of few rows keep all digits: every result of a product is hi + lo, every
// product of two has three passes (hi hi, hi lo, lo hi).  A few rows do not average
// roundings out: u of 4 to 16 was off by up to 6.5 10^-3 of itself, of 17 to 32 by 2.9,
// of more by at most 1.9; with them it is 0.4.  They are no gift (48 x 80, a launch for
// each product: 85.7 us a call with passes and lo's, 70.5 without), hence 32.  The Gram matrix of longer rows takes
// one pass: it averages over them.
constexpr int64_t kPrecise = 32, kPreciseGram = 512;
inline bool is_precise(int64_t m) { return m <= kPrecise; }

// What a k-block of a 256 x 128 tile takes next to one of 256 x 256, and a tile's
// epilogue that no product hides, in k-blocks.
constexpr double kNarrowBlock = 0.65, kTileBlocks = 4.0;

// Deals n units of a cost to the pairs, least loaded first: windows of neighbouring
// pairs with the same load.  A deal takes a segment a step, of which windows whose loads
// do not meet take many, so each leaves one to every deal behind it.
struct Dealer {
    struct Window {
        int from, len;
        double load;
    };
    Window w[2 * kMaxSegments];
    int windows = 1;
    double most = 0;
    Dealer(int pairs) { w[0] = {0, pairs, 0}; }

    // `behind`: the deals still to come.
    void deal(Tiles *p, int first, int n, double cost, int behind) {
        int u = first;
        const int end = first + n;
        while (u < end) {
            if (p->segments >= kMaxSegments - 1 - behind || windows >= 2 * kMaxSegments - 1) {  // the rest in turn
                int all = 0;
                for (int i = 0; i < windows; ++i) all += w[i].len;
                segment(p, u, end, 0, all);
                most += cost * ((end - u + all - 1) / all);
                return;
            }
            int low = 0;
            double next = INFINITY;
            for (int i = 1; i < windows; ++i)
                if (w[i].load < w[low].load) low = i;
            for (int i = 0; i < windows; ++i)
                if (i != low) next = std::min(next, w[i].load);
            Window &x = w[low];
            const double rounds_most = std::isfinite(next) ? std::max(1.0, std::ceil((next - x.load) / cost - 1e-9)) : 1e9;
            const int rounds = static_cast<int>(std::min<double>(rounds_most, (end - u) / x.len));
            if (rounds > 0) {
                segment(p, u, u + rounds * x.len, x.from, x.len);
                u += rounds * x.len;
                x.load += rounds * cost;
                most = std::max(most, x.load);
            } else {  // fewer than a round: the window splits
                const int rem = end - u;
                segment(p, u, end, x.from, rem);
                for (int i = windows; i > low + 1; --i) w[i] = w[i - 1];
                ++windows;
                w[low + 1] = {x.from + rem, x.len - rem, x.load};
                w[low].len = rem;
                w[low].load += cost;
                most = std::max(most, w[low].load);
                u = end;
            }
            for (int i = 0; i + 1 < windows;) {  // neighbours that are level become one
                if (std::fabs(w[i].load - w[i + 1].load) < 1e-9 * cost) {
                    w[i].len += w[i + 1].len;
                    for (int j = i + 1; j + 1 < windows; ++j) w[j] = w[j + 1];
                    --windows;
                } else {
                    ++i;
                }
            }
        }
    }
    void segment(Tiles *p, int from, int to, int pair0, int pairs) {
        if (p->segments >= kMaxSegments) {  // (never)
            most = INFINITY;
            return;
        }
        const int s = p->segments++;
        p->from[s] = from;
        p->to[s] = to;
        p->pair0[s] = static_cast<int16_t>(pair0);
        p->pairs[s] = static_cast<int16_t>(pairs);
    }
};

// Tiles of 256 x bn, dealt to the pairs; returns what the longest-working pair has
// to do, in k-blocks of 256 x 256, or infinity where the tiles could not all be dealt.
inline double deal(const Chunk &c, int pairs, Tiles *p, int form, int bn) {
    *p = Tiles{};
    p->bn = bn;
    Dealer dealer(pairs);
    int order[kMaxClasses], n[kMaxClasses];
    for (int k = 0; k < c.classes; ++k) {
        const int64_t m = c.shape[k].m, cols = form == kTimesX ? c.shape[k].n : m;
        const int64_t tm = (m + 255) / 256, tn = (cols + bn - 1) / bn;
        int64_t per = tm * tn;
        if (form == kGram || form == kSquareSym) {
            per = 0;
            for (int64_t i = 0; i < tm; ++i) per += tn - 256 / bn * i;
        }
        order[k] = k;
        n[k] = static_cast<int>(per) * (c.first[k + 1] - c.first[k]);
        p->unit0[k] = p->units;
        p->units += n[k];
        p->per[k] = static_cast<int>(per);
        p->tiles_m[k] = static_cast<int>(tm);
        p->tiles_n[k] = static_cast<int>(tn);
        p->rows[k] = static_cast<int>(m);
        p->cols[k] = static_cast<int>(cols);
        p->kb[k] = static_cast<int>(((form == kGram ? c.shape[k].n : m) + kBK - 1) / kBK);
        p->first[k] = c.first[k];
    }
    p->classes = c.classes;
    p->unit0[c.classes] = p->units;
    sort_few(order, c.classes, [&](int a, int b) { return p->kb[a] != p->kb[b] ? p->kb[a] > p->kb[b] : a < b; });
    const double block_cost = bn == 256 ? 1.0 : kNarrowBlock;
    for (int i = 0; i < c.classes; ++i)
        dealer.deal(p, p->unit0[order[i]], n[order[i]],
                    block_cost * (p->kb[order[i]] * (is_precise(c.shape[order[i]].m) ? 3 : 1) + kTileBlocks),
                    c.classes - 1 - i);
    return dealer.most;
}

// Whether a pair of CTAs for each matrix is faster than a launch for each product, by
// what both were measured to take (us): a launch 2.75, and 0.25 for each 64 rows; the
// long rows of the Gram matrix; where there are many, a good part of what a pair would
// have taken by itself.  Five steps on one [128, 128] 43 and 68, on [256, 256] 68 and 75,
// on [128, 1536] 82 and 79, on 64 of them 134 and 170, on [256, 1536] 117 and 85, on 64 of
// them 210 and 260.
inline bool small_pays(const Chunk &c, int pairs, int n_steps) {
    const int products = 7 * (n_steps / 2) + 3 * (n_steps % 2), turns = (n_steps + 1) / 2;
    double launches = 0, all = 0, longest = 0;
    for (int k = 0, at = 0; k < c.classes; ++k) {
        const int64_t m = c.shape[k].m, units = c.first[k + 1] - c.first[k];
        if (m > kSmallMost) return false;
        const double kb_m = static_cast<double>((m + kBK - 1) / kBK), kb_n = static_cast<double>((c.shape[k].n + kBK - 1) / kBK);
        const double passes = is_precise(m) ? 1.2 : 1.0;
        const double one = passes * (products * (1.24 + 0.476 * kb_m) + turns * (0.5 + 0.065 * kb_m) * kb_n);
        launches = std::max(launches, passes * (products * (2.75 + 0.25 * kb_m) + turns * 0.17 * kb_n));
        all += one * static_cast<double>(units);
        for (int64_t i = 0; i < units; ++i, ++at)  // (dealt in turn, the longest first)
            if (at % pairs == 0) longest += one;
    }
    return longest < launches + 0.8 * all / pairs;
}

}  // namespace puro
