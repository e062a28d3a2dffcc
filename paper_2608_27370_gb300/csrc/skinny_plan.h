// skinny_plan.h -- how many warps a block of the linears of a few tokens has
// (see skinny.cu).  Host code without a CUDA call.
#pragma once

#include <cstdint>

namespace puro {

constexpr int kSkinnyForms = 5;
constexpr int kSkinnyWarps[kSkinnyForms] = {16, 8, 6, 12, 4};  // a block, by form

// The form for `blocks` blocks that each reduce over `steps` steps of 32 k, a
// warp `unroll` of them at a time, where resident[i] blocks of form i are
// resident at once: the fewest loads that follow one another, which is rounds
// of blocks times rounds of a warp's steps.  Of equal ones that with the
// fewest rounds of blocks, then the first; four warps, which keep the fewest
// loads in flight, only where nothing equals them.
inline int skinny_form(int64_t blocks, int64_t steps, int unroll, const int64_t (&resident)[kSkinnyForms]) {
    auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    int best = 0;
    int64_t least = INT64_MAX, fewest = INT64_MAX;
    for (int i = 0; i < kSkinnyForms; ++i) {
        if (resident[i] <= 0) continue;
        const int64_t waves = ceil_div(blocks, resident[i]), rounds = waves * ceil_div(ceil_div(steps, kSkinnyWarps[i]), unroll);
        if (rounds < least || (rounds == least && waves < fewest && kSkinnyWarps[i] > 4)) {
            best = i;
            least = rounds;
            fewest = waves;
        }
    }
    return best;
}

}  // namespace puro
