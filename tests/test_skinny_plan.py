"""csrc/skinny_plan.h: the warps a block of the linears of a few tokens."""
import os
import subprocess

import pytest

import paper_2608_27370_gb300 as P

SOURCE = r"""
#include <cstdio>
#include "skinny_plan.h"
int main() {
    long long b, s, r[5];
    int u;
    while (std::scanf("%lld %lld %d %lld %lld %lld %lld %lld", &b, &s, &u, r, r + 1, r + 2, r + 3, r + 4) == 8) {
        const int64_t resident[5] = {r[0], r[1], r[2], r[3], r[4]};
        std::printf("%d\n", puro::kSkinnyWarps[puro::skinny_form(b, s, u, resident)]);
    }
}
"""
WARPS = (16, 8, 6, 12, 4)
LINEAR, GATED = ((304, 760, 912, 608, 1520), 3), ((304, 608, 912, 456, 1368), 2)  # resident blocks on 152 SMs, steps at once


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    src, exe = folder / "plan.cpp", str(folder / "plan")
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", P._build.CSRC, str(src), "-o", exe], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, (n // 8, -(-k // 32), unroll, *resident))) for n, k, (resident, unroll) in cases)
        return [int(x) for x in subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.split()]
    return run


def _rounds(n, k, kind, warps):
    resident, unroll = kind
    waves = -(-(n // 8) // resident[WARPS.index(warps)])
    return waves * -(-(-(-(-(-k // 32)) // warps)) // unroll), waves


def test_no_form_has_fewer_rounds(plan):
    cases = [(n, k, kind) for n in list(range(8, 4000, 152)) + list(range(4000, 40000, 1096)) for k in (8, 512, 1536, 2048, 8960)
             for kind in (LINEAR, GATED)]
    for (n, k, kind), w in zip(cases, plan(cases)):
        mine = _rounds(n, k, kind, w)
        for other in WARPS:
            theirs = _rounds(n, k, kind, other)
            assert mine[0] <= theirs[0] and (mine <= theirs or 4 in (other, w)), (n, k, kind, w, other)
            assert w != 4 or other == 4 or mine[0] < theirs[0], (n, k, kind)


def test_neighbouring_widths_take_one_form(plan):
    """8960 and the widths behind it are as many rounds of blocks: a rule by 6800 or 9300 warps in all, just above what
    8960 columns take, gave a linear of 9072 columns another form than one of 8960, and both of them a slower one."""
    for kind in (LINEAR, GATED):
        assert set(plan([(n, 1536, kind) for n in (8192, 8960, 9064, 9072, 9216, 9728)])) == {8}


def test_a_form_whose_blocks_cannot_be_counted_is_not_taken(plan):
    for i, w in enumerate(WARPS):
        only = tuple(300 if j == i else 0 for j in range(5))
        assert plan([(2048, 1536, (only, 2))]) == [w]
