"""Keys of the paged attention go from the lanes that load them to the lanes that multiply them through LDS, without a barrier: what tells the
compiler to keep their order is in the code that it makes, without a GPU."""
import os
import re
import subprocess

from paper_2601_11676_amd import build

SOURCE = """
#include "paged_attention.hpp"
namespace halo { namespace {
template <typename Core>
__global__ __launch_bounds__(64) void turn_twice(AttendArgs a)
{
    __shared__ __align__(16) char own[Core::kStage];
    Core core;
    core.place(a.D, threadIdx.x, own);
    auto *rows = reinterpret_cast<u32x4 *>(const_cast<void *>(a.k));
    for (int turn = 0; turn < 2; ++turn) {
        for (int i = 0; i < Core::kSub; ++i)
            for (int s = 0; s < Core::KS; ++s) core.kf[i][s] = __builtin_bit_cast(std::remove_reference_t<decltype(core.kf[i][s])>, rows[(i * Core::KS + s) * 64 + threadIdx.x]);
        turn_keys(core);
        for (int i = 0; i < Core::kSub; ++i)
            for (int s = 0; s < Core::KS; ++s) rows[(i * Core::KS + s) * 64 + threadIdx.x] = __builtin_bit_cast(u32x4, core.kf[i][s]);
    }
}
}
void go(const AttendArgs &a)
{
    turn_twice<CoreBf16One<64, true, kKeepAll>><<<1, 64>>>(a);
    turn_twice<CoreBf16One<128, false, kKeepAll>><<<1, 64>>>(a);
    turn_twice<CoreF32Few<64, true, kKeepAll>><<<1, 64>>>(a);
    turn_twice<CoreF32Two<128, true, kPassBoth>><<<1, 64>>>(a);
}
}
"""


def test_lanes_that_use_each_others_keys_are_kept_in_order(tmp_path):
    source, out = tmp_path / "turn.hip", tmp_path / "turn.ll"
    source.write_text(SOURCE)
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-Wall", "-Wextra")]
    subprocess.run(["hipcc", *flags, "-I", build.CSRC, "--cuda-device-only", "-S", "-emit-llvm", "-o", str(out), str(source)], check=True,
                   timeout=120)
    kernels = re.findall(r"define [^\n]*amdgpu_kernel[^\n]*turn_twice(.*?)\n}", out.read_text(), re.S)
    assert len(kernels) == 4
    for text in kernels:
        order = ""
        for line in text.split("\n"):
            if "addrspace(3)" in line and re.match(r"\s*store ", line):
                order += "S"
            elif "addrspace(3)" in line and re.search(r"= load ", line):
                order += "L"
            elif re.match(r'\s*fence syncscope\("wavefront"\) acq_rel', line):
                order += "F"
            elif "wave.barrier" in line:
                order += "B"
        # the two turns one after the other, or one in a loop
        assert re.fullmatch(r"(S+FBL+FB){1,2}", order), order
