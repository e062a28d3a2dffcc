"""What of a table of Muon directions may lie in the same place (no GPU)."""
import random
import subprocess

import pytest

import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import _build
from test_muon_reference import A, BAD, call, entry, table

# Reads tables of "count", then per matrix "rows cols  grad stride type  momentum  u stride type", and prints whether writes overlap.
SOURCE = r"""
#include <cstdio>
#include <vector>
#include "muon_plan.h"
using namespace puro;
int main() {
    int count;
    while (std::scanf("%d", &count) == 1) {
        std::vector<puro_muon_matrix_t> mats(count);
        for (auto &m : mats) {
            long long r, c, g, gs, v, u, us;
            if (std::scanf("%lld %lld %lld %lld %d %lld %lld %lld %d", &r, &c, &g, &gs, &m.grad_type, &v, &u, &us, &m.u_type) != 9) return 1;
            m.rows = r, m.cols = c, m.grad_stride = gs, m.u_stride = us;
            m.grad = reinterpret_cast<const void *>(g), m.momentum = reinterpret_cast<float *>(v), m.u = reinterpret_cast<void *>(u);
        }
        std::vector<Place> places(3 * count);
        std::printf("%d\n", writes_overlap(mats.data(), count, places.data()));
    }
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    folder = tmp_path_factory.mktemp("overlap")
    src, exe = folder / "overlap.cpp", str(folder / "overlap")
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", _build.CSRC, "-I", _build.INCLUDE, str(src), "-o", exe], check=True)

    def run(tables):
        text = "\n".join(" ".join(map(str, [len(t)] + [x for m in t for x in m])) for t in tables)
        return [bool(int(x)) for x in subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.split()]
    return run


def byte_sets(m):
    """Of (rows, cols, grad, stride, type, momentum, u, stride, type): what the gradient, the momentum and u are."""
    r, c, g, gs, gt, v, u, us, ut = m

    def of(at, stride, size):
        return {at + (i * stride + j) * size + b for i in range(r) for j in range(c) for b in range(size)} if at else set()
    return of(g, gs, 4 if gt else 2), of(v, c, 4), of(u, us, 4 if ut else 2)


def expected(t):
    sets = [byte_sets(m) for m in t]
    for i, (g, v, u) in enumerate(sets):
        if v & (g | u):
            return True
        for j, (h, w, y) in enumerate(sets):
            if i != j and (v & (h | w | y) or u & (h | w | y)):
                return True
    return False


def test_random_tables_against_their_bytes(overlap):
    """Views of one small piece of memory, of any strides; of a wider matrix's columns; a stride of 0."""
    rng, tables = random.Random(1), []
    for _ in range(6000):
        t, wide = [], rng.choice((0, 8, 12))  # columns of one wide matrix, or anything
        room = rng.choice((200, 600, 2400))

        def at():
            return 4096 + 4 * rng.randrange(room // 4)
        for _ in range(rng.randint(1, 3)):
            r, c = rng.choice((0, 1, 2, 3, 5)), rng.randint(1, 5)
            gs = wide or rng.choice((0, 1, c, c + rng.randint(0, 9)))
            us = wide or c + rng.randint(0, 9)
            t.append((r, c, at(), gs, rng.randint(0, 1), at() if rng.random() < 0.4 else 0, at(), us, rng.randint(0, 1)))
        tables.append(t)
    want = [expected(t) for t in tables]
    assert 1000 < sum(want) < 5500
    for t, got, w in zip(tables, overlap(tables), want):
        assert got == w, t


def test_large_strides_and_many_slices(overlap):
    wide = [(1 << 20, 16, 1 << 44, 4096, 1, 0, (1 << 40) + 64 * i, 4096, 1) for i in range(64)]  # 64 columns blocks of one matrix of 16 GiB
    far = (1 << 20, 1 << 20, 1 << 30, 1 << 62, 1, 0, 1 << 50, 1 << 62, 1)
    assert overlap([wide, wide + [(1, 1, 1 << 45, 1, 1, 0, (1 << 40) + (1 << 33) + 4, 1, 0)], [far]]) == [False, True, False]


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return P.load_library()


def test_the_entry_point_refuses(lib):
    B, C, D, E = (A + (i << 22) for i in range(1, 5))
    first = dict(grad=A, momentum=B, u=C)
    for one, other in ((dict(grad=B), dict()), (dict(u=B), dict()), (dict(grad=B + 1024), dict()), (dict(), dict(momentum=B)), (dict(), dict(momentum=B + 4)),
                       (dict(), dict(u=C)), (dict(), dict(u=C + 64)), (dict(), dict(u=B)), (dict(), dict(u=A)), (dict(), dict(grad=C, gt=0)),
                       (dict(), dict(grad=B)), (dict(momentum=None), dict(u=A))):
        assert call(lib, table(entry(**{**first, **one}), entry(**{**dict(grad=A, momentum=D, u=E), **other}))) == BAD, (one, other)
    assert call(lib, table(entry(grad=A, momentum=A, u=C))) == BAD
