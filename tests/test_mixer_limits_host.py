"""Sizes past what a launch can hold (2^32 threads) are refused before the first launch of a call, without a GPU: none of these calls touches its
pointers.  And plans at the largest sizes, in which no sum of 32 bits overflows."""
import ctypes
import os
import subprocess

from paper_2404_07904_amd import binding
from test_mixer_host import BIG, E_NULL, E_UNSUP, FAKE, FAKE_WS, ROOT, conv, conv_bwd, conv_fwd, ssm, ssm_bwd, ssm_fwd


def test_convolution():
    # waves of 4 or 16 tokens and 512 channels in bf16, four to a workgroup: fewer than 2^24 workgroups
    most = (1 << 24) * 4 * 16 - 64
    assert conv_fwd(conv(B=1, N=most + 64, D=8)) == E_UNSUP and conv_fwd(conv(B=1, N=most, D=8), x=None) == E_NULL
    assert conv_fwd(conv(B=1, N=1 << 28, D=1)) == E_UNSUP
    # sequences' states: 256 vectors a workgroup on top
    assert conv_fwd(conv(B=1 << 30, N=1, D=1), fin=FAKE) == E_UNSUP
    for bad in (conv(B=1, N=0x7fffff00, D=4000), conv(B=1, N=4, D=1 << 30, K=4)):
        assert conv_bwd(bad) == E_UNSUP
        assert binding.lib().hgrn2_conv_bwd_workspace_bytes(ctypes.byref(bad), 0) == 0
    assert conv_bwd(conv(B=1, N=1 << 20, D=4096), gy=None) == E_NULL


def test_scan():
    # one workgroup for 64 channels of a sequence
    assert ssm_fwd(ssm(B=1 << 18, N=1, D=4096)) == E_UNSUP and ssm_fwd(ssm(B=(1 << 18) - 1, N=1, D=4096), x=None) == E_NULL
    assert binding.lib().hgrn2_ssm_fwd_workspace_bytes(ctypes.byref(ssm(B=1 << 18, N=1, D=4096)), 0) == 0
    # a thread for every element of grad_B, grad_C and the parameters' gradients
    wide = ssm(B=1, N=1 << 26, D=64, S=32)
    assert ssm_bwd(wide) == E_UNSUP and binding.lib().hgrn2_ssm_bwd_workspace_bytes(ctypes.byref(wide), 0, 0) == 0
    assert ssm_fwd(wide, x=None) == E_NULL
    assert ssm_bwd(ssm(B=1, N=(1 << 26) - 100, D=64, S=32), gy=None) == E_NULL
    step = binding.lib().hgrn2_ssm_step

    def one(B, D, x=FAKE):
        return step(ctypes.byref(ssm(B=B, N=1, D=D)), x, FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, None)

    assert one(1 << 18, 4096) == one(1 << 14, 1 << 16) == E_UNSUP and one(1 << 17, 4096, x=None) == E_NULL


def test_quantisation_and_product():
    L = binding.lib()

    def quant(M, K, qt=None, x=FAKE):
        return L.hgrn2_quant8(M, K, 1, x, 0, 1, FAKE, FAKE, qt, qt, None)

    assert quant(1 << 28, 1) == E_UNSUP and quant((1 << 28) - 16, 1, x=None) == E_NULL
    assert quant(0x7fffff00, 129, qt=FAKE) == E_UNSUP and quant(1 << 30, 100, qt=FAKE, x=None) == E_NULL

    def proj(M, N, K=128, out=1, a=FAKE):
        return L.hgrn2_proj8(M, N, K, a, FAKE, 1, FAKE, FAKE, 1, None, 0, out, FAKE, FAKE_WS, BIG, None)

    assert proj(1, 1 << 27) == E_UNSUP and proj(1, (1 << 27) - 16, a=None) == E_NULL
    assert proj(1 << 25, 1 << 13, K=2048, a=None) == E_NULL and proj(1 << 27, 1 << 13, K=2048) == proj(1 << 28, 1 << 15) == E_UNSUP


PLAN = r"""
#include <cstdio>
#include <initializer_list>
#include "ssm_plan.hpp"
using namespace hgrn2;
int main()
{
    for (int N : {1 << 30, (1 << 30) + 16, 0x7fffffff - 64})
        for (int S : {8, 16, 32})
            for (int D : {1, 4096})
                for (int way = 0; way < 4; ++way) {
                    const SsmPlan p = ssm_plan(1, N, D, S, 1, way == 1, way == 0, way == 2);
                    if (p.runs < 1 || (long long)p.runs * p.len < N || (long long)(p.runs - 1) * p.len >= N || (way == 0 && p.runs != 1)) return 1;
                    if (p.chunks != (int)(((long long)N + ssm_chunk(S) - 1) / ssm_chunk(S)) || p.total != p.runs) return 1;
                }
    std::puts("ok");
}
"""


def test_plans_of_the_longest_sequences(tmp_path):
    (tmp_path / "plan.cpp").write_text(PLAN)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover", "-static-libubsan",
                           "-I", os.path.join(ROOT, "paper_2404_07904_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", str(tmp_path / "plan")])
    assert subprocess.check_output([str(tmp_path / "plan")], text=True).strip() == "ok"
