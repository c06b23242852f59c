"""Which kernel of the 8-bit product the sizes of its GPU tests take (csrc/proj8_plan.hpp, compiled here by the host compiler, no GPU needed): every tile with
a ring of steps that goes round several times and a last group of scales that is not whole, alone and in shares, for either type of results."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# M, N, K and what a product with bf16 and with fp32 results takes: tile (0: the kernel for few rows), shares
SIZES = [(16, 33, 1200, (0, 1), (0, 1)), (30, 500, 2100, (0, 1), (0, 1)), (64, 80, 3900, (0, 1), (0, 1)), (64, 8000, 8000, (64, 2), (64, 2)),
         (700, 1000, 1900, (64, 1), (64, 1)), (96, 80, 16600, (64, 16), (64, 16)), (1025, 2049, 2100, (128, 1), (128, 1)),
         (513, 2000, 8000, (128, 2), (128, 2)), (4000, 3900, 1200, (256, 1), (256, 1)), (1000, 1050, 16200, (128, 2), (256, 8)),
         (2800, 2700, 8000, (128, 1), (256, 2)), (768, 700, 65400, (256, 16), (256, 16))]
PLAN = r"""
#include <cstdio>
#include <cstdlib>
#include "proj8_plan.hpp"
int main(int, char** a)
{
    const int M = std::atoi(a[1]), N = std::atoi(a[2]), K = std::atoi(a[3]);
    for (bool exact : {false, true}) {
        const hgrn2::Proj8Plan p = hgrn2::plan_proj8(M, N, (K + 127) / 128, exact);
        std::printf("%d %d ", p.tile, p.splits);
    }
}
"""


def test_sizes_of_the_gpu_tests(tmp_path):
    (tmp_path / "plan.cpp").write_text("#include <initializer_list>\n" + PLAN)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2404_07904_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")])
    for M, N, K, bf16, fp32 in SIZES:
        got = [int(v) for v in subprocess.check_output([str(tmp_path / "plan"), str(M), str(N), str(K)], text=True).split()]
        assert got == [*bf16, *fp32], (M, N, K, got)
        # a share has more steps than any ring has places (8, 4, 2 for 64, 128, 256), and the last group of four is not whole
        for tile, shares in (bf16, fp32):
            assert tile == 0 or -(-K // 128) // shares >= 8
        assert -(-K // 128) % 4 != 0
