"""Reset marks of a lane's eight steps shifted into place at the end of a row, for rows up to the longest that is accepted: csrc/ss_gate.hip
compiled for the host, with signed overflow trapped."""
import ctypes
import os
import subprocess

from paper_2312_00752_amd import binding as B
from paper_2312_00752_amd import build

PROGRAM = r"""
#include <cstdio>
#include "ss_gate.hip"
int main()
{
    const long lengths[] = {8, 9, 15, 16, 100, 4097, (1l << 28) - 1, (1l << 28) + 8, (1l << 28) + 13, (1l << 30) + 3, 0x7fffffffl - 4 * ss::GATE_PIECE};
    for (const long L : lengths)
        for (const long base : {0l, 8l, L / 16 * 8, L - L % 8 - 16, L - L % 8 - 8, L - L % 8, L - L % 8 + 8, L - L % 8 + 1600}) {
            if (base < 0) continue;
            // marks as they stand from min(base, L - 8) on: the place of each step, of which those of the slice are wanted
            const long from = base < L - 8 ? base : L - 8;
            uint32_t w[2] = {0, 0}, want[2] = {0, 0};
            for (int j = 0; j < 8; ++j) {
                w[j / 4] |= (uint32_t)(from + j) % 251 + 1 << 8 * (j % 4);
                if (base + j < L) want[j / 4] |= (uint32_t)(base + j) % 251 + 1 << 8 * (j % 4);
            }
            const uint2 got = ss::marks_settle(make_uint2(w[0], w[1]), (int)base, (int)L);
            if (got.x != want[0] || got.y != want[1]) {
                std::printf("length %ld, slice at %ld: %08x %08x, not %08x %08x\n", L, base, got.x, got.y, want[0], want[1]);
                return 1;
            }
        }
    std::printf("done\n");
    return 0;
}
"""


def test_marks_of_long_rows(tmp_path):
    source, obj, program = (str(tmp_path / n) for n in ("marks.hip", "marks.o", "marks"))
    head = "#include <hip/hip_runtime.h>\n#undef __global__\n#define __global__ __device__\n#undef __launch_bounds__\n#define __launch_bounds__(...)\n" \
           "#undef hipLaunchKernelGGL\n#define hipLaunchKernelGGL(...)\n#define hipGetLastError() hipSuccess\n"
    with open(source, "w") as f:
        f.write(head + PROGRAM)
    subprocess.run([build._hipcc(), "--offload-arch=gfx950", "-std=c++17", "-O0", "-ftrapv", "-fPIC", "--offload-host-only", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), "-c", source, "-o", obj], check=True, capture_output=True)
    subprocess.run(["g++", obj, "-o", program], check=True, capture_output=True)
    out = subprocess.run([program], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "done\n", (out.returncode, out.stdout)


def test_steps_past_the_longest_row():
    """The last round of a team of four may lie up to three pieces of 512 steps behind the row; its steps are numbered in 32 bits too, so a row
    that leaves no room for them is refused."""
    p = B.GateParams()
    p.batch = p.dim = 1
    p.io_dtype = B.SS_BF16
    p.flags = B.SS_GATE_SAVE_FOR_BWD
    for f in ("x", "f", "rate", "out"):
        setattr(p, f, 1 << 20)
    for seqlen, code in ((2 ** 31 - 1 - 2 * 512, B.SS_ERR_UNSUPPORTED), (2 ** 31 - 1 - 2039, B.SS_ERR_UNSUPPORTED), (2 ** 31 - 1 - 2048, B.SS_ERR_WORKSPACE)):
        p.seqlen = seqlen
        last = -(-seqlen // 512) - 1 + 3   # piece
        if code != B.SS_ERR_UNSUPPORTED:
            assert last * 512 + 64 * 8 < 2 ** 31
        assert B.lib().ss_gate_fwd(ctypes.byref(p), None) == code, seqlen
