"""csrc/muon_plan.h: who takes the tiles of the Muon directions' products."""
import random
import subprocess

import pytest

import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import workloads as W

# Reads tables "pairs count  m n  m n ..." and walks, as the kernels do, all pairs through the tiles of every product's form and width, chunk by
# chunk.  Of each table: chunks, the most segments, tiles that no pair takes, that several take, that lie where another does, whether
# anything behind the tiles was written, and whether a pair has more to do than deal() says.
SOURCE = r"""
#include <cstdio>
#include <cstring>
#include <set>
#include <tuple>
#include <vector>
#include "muon_plan.h"
using namespace puro;
struct Guarded {
    Tiles t;
    unsigned char behind[4096];
};
template <int BN, bool SYM>
long misplaced(const Tiles &t, const Chunk &c) {
    std::set<std::tuple<int, int, int, int>> at;
    long bad = 0;
    for (int u = 0; u < t.units; ++u) {
        const Unit w = unit_of<BN, SYM>(t, u);
        const bool in = w.z >= 0 && w.z < c.first[w.cls + 1] - c.first[w.cls] && w.m0 < t.rows[w.cls] && w.n0 < t.cols[w.cls] && (!SYM || w.n0 >= w.m0);
        bad += !in || !at.insert({w.cls, w.z, w.m0, w.n0}).second;
    }
    return bad;
}
int main() {
    int pairs, count;
    static Guarded g;
    while (std::scanf("%d %d", &pairs, &count) == 2) {
        std::vector<puro_muon_matrix_t> mats(count);
        for (auto &m : mats) {
            long long r, c;
            if (std::scanf("%lld %lld", &r, &c) != 2) return 1;
            m.rows = r;
            m.cols = c;
        }
        long chunks = 0, segments = 0, missed = 0, twice = 0, bad = 0, behind = 0, more = 0;
        for (int at = 0; at < count;) {
            Chunk c;
            at = take_chunk(mats.data(), at, count, &c);
            ++chunks;
            for (int form = 0; form < kForms; ++form)
                for (int bn : {256, 128}) {
                    std::memset(&g, 0x5A, sizeof g);
                    const double most = deal(c, pairs, &g.t, form, bn);
                    const Tiles &t = g.t;
                    for (unsigned char b : g.behind) behind += b != 0x5A;
                    segments = std::max<long>(segments, t.segments);
                    std::vector<int> taken(t.units);
                    for (int pair = 0; pair < std::min(t.units, pairs); ++pair) {
                        Walk w;
                        double load = 0;
                        for (int u; (u = w.next(t, pair)) >= 0;) {
                            if (u >= t.units || ++taken[u] > 2) break;
                            const int k = bn == 256 ? unit_of<256, false>(t, u).cls : unit_of<128, false>(t, u).cls;
                            load += (bn == 256 ? 1.0 : kNarrowBlock) * (t.kb[k] * (is_precise(c.shape[k].m) ? 3 : 1) + kTileBlocks);
                        }
                        more += !(load <= most * (1 + 1e-9));
                    }
                    for (int x : taken) {
                        missed += x == 0;
                        twice += x > 1;
                    }
                    const bool sym = form == kGram || form == kSquareSym;
                    bad += bn == 256 ? sym ? misplaced<256, true>(t, c) : misplaced<256, false>(t, c)
                                     : sym ? misplaced<128, true>(t, c) : misplaced<128, false>(t, c);
                }
        }
        std::printf("%ld %ld %ld %ld %ld %ld %ld\n", chunks, segments, missed, twice, bad, behind, more);
    }
}
"""
PAIRS = 76


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    src, exe = folder / "plan.cpp", str(folder / "plan")
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", P._build.CSRC, "-I", P._build.INCLUDE, str(src), "-o", exe], check=True)

    def run(tables):
        """tables: (pairs, [(count, m, n), ...])."""
        lines = []
        for pairs, shapes in tables:
            mats = [(m, n) for count, m, n in shapes for _ in range(count)]
            lines.append(" ".join(map(str, [pairs, len(mats)] + [x for s in mats for x in s])))
        out = subprocess.run([exe], input="\n".join(lines), check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
        assert len(out) == len(tables)
        return [tuple(map(int, x.split())) for x in out]
    return run


def each_tile_once(plan, tables):
    for table, (chunks, segments, *wrong) in zip(tables, plan(tables)):
        assert wrong == [0, 0, 0, 0, 0], (table, segments, wrong)


def layer(linears, apart, heads):
    """One layer's matrices, the fused projections whole or in their parts."""
    out = []
    for name, n, k in linears:
        if apart and name == "qkv":
            q, kv, d = heads
            out += [(1, q * d, k), (2, kv * d, k)]
        elif apart and name == "gate_up":
            out.append((2, n // 2, k))
        else:
            out.append((1, n, k))
    return out


@pytest.mark.parametrize("linears,heads", [(W.QWEN2_1P5B_LINEARS, (12, 2, 128)), (W.QWEN3_1P7B_LINEARS, (16, 8, 128))])
@pytest.mark.parametrize("apart", [False, True])
def test_the_frameworks_own_layers(plan, linears, heads, apart):
    each_tile_once(plan, [(PAIRS, layer(linears, apart, heads) * n) for n in range(1, 29)])


def test_tables_that_filled_the_segments(plan):
    each_tile_once(plan, [(PAIRS, t) for t in (
        [(25, 40, 40), (1, 512, 512), (3, 384, 768), (26, 288, 2048)],
        [(8, 1507, 2042), (9, 1363, 4466), (8, 88, 1143)],
        [(11, 3185, 3338), (8, 6, 147), (7, 362, 4466)],
        [(2, 1024, 1664), (6, 384, 2816), (1, 256, 1152), (5, 512, 768), (3, 128, 1280), (4, 128, 2944)],
        [(10, 32, 80), (10, 3496, 874), (10, 1368, 1296)],
        [(2, 4096, 4096), (2, 1024, 4096), (2, 4096, 6144), (2, 14336, 4096)] * 2)])


@pytest.mark.parametrize("most", [1, 3, 8, 12])
def test_random_tables(plan, most):
    """Of up to `most` shapes, on any number of pairs."""
    rng = random.Random(most)

    def size():
        return int(4 * 1536 ** rng.random()) if rng.random() < 0.7 else 160 * rng.randint(1, 32)
    tables = []
    for _ in range(250):
        shapes = [(rng.choice((1, 1, 2, 3, 5, 12, 30)), size(), size()) for _ in range(rng.randint(1, most))]
        tables.append((rng.choice((PAIRS, PAIRS, 74, 66, 7, 1)), shapes))
    each_tile_once(plan, tables)


def test_one_shape_of_any_number(plan):
    each_tile_once(plan, [(PAIRS, [(count, m, n)]) for m, n in ((1, 1), (257, 300), (1536, 1536), (700, 9000)) for count in (1, 2, 75, 76, 77, 128, 129, 300)])
