"""csrc/register_check.h against made-up queries: what a failed one answers, and what is kept."""
import os
import subprocess

import paper_2608_27370_gb300 as P

SOURCE = r"""
#include <cstdio>
#include "register_check.h"
int main() {
    puro::RegisterCheck check;
    int asked = 0;
    auto ask = [&](int device, cudaError_t e, int regs) {
        const cudaError_t r = check.enough(device, 20, 1888, [&](int *out) { ++asked; *out = regs; return e; });
        std::printf("%d %d\n", static_cast<int>(r), asked);
    };
    ask(0, cudaErrorMemoryAllocation, 0);   // a query that fails once
    ask(0, cudaErrorMemoryAllocation, 96);
    ask(0, cudaSuccess, 96);                // 1920 registers
    ask(0, cudaErrorMemoryAllocation, 0);   // not asked again
    ask(1, cudaErrorInvalidDevice, 0);      // another device
    ask(1, cudaSuccess, 94);                // 1880
    ask(1, cudaSuccess, 96);
    ask(0, cudaSuccess, 0);
    ask(64, cudaSuccess, 96);               // one that nothing is kept for
    ask(64, cudaSuccess, 94);
    ask(-1, cudaSuccess, 96);
}
"""
SUCCESS, NO_MEMORY, NO_DEVICE, TOO_FEW = 0, 2, 101, 701


def test_only_a_query_that_succeeded_is_kept(tmp_path):
    src, exe = tmp_path / "check.cpp", str(tmp_path / "check")
    src.write_text(SOURCE)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(P._build._nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", P._build.CSRC, "-isystem", cuda, str(src), "-o", exe], check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    assert [tuple(map(int, x.split())) for x in lines] == [
        (NO_MEMORY, 1), (NO_MEMORY, 2), (SUCCESS, 3), (SUCCESS, 3), (NO_DEVICE, 4), (TOO_FEW, 5), (TOO_FEW, 5), (SUCCESS, 5),
        (SUCCESS, 6), (TOO_FEW, 7), (SUCCESS, 8)]
