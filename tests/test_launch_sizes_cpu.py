"""What the entry points launch, over sizes up to what a card's memory holds: every launch within what a launch can be, and nothing launched
by a call that is refused.  The entry points of a source file run on the host with the launches recorded instead of made."""
import os
import subprocess

import pytest

from paper_2312_00752_amd import build

HEAD = r"""
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <vector>
struct Launch { dim3 grid, block; };
static std::vector<Launch> launches;
#undef __global__
#define __global__ __device__
#undef __launch_bounds__
#define __launch_bounds__(...)
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) launches.push_back({grid, block})
#define hipGetLastError() hipSuccess
#include "SOURCE"

static uint64_t seed = 1;
static double uniform() { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return (double)(seed >> 11) / 9007199254740992.0; }
static int32_t any(double most)   // up to `most`, spread over the logarithm; now and then the end itself
{
    return uniform() < 0.1 ? (int32_t)most : (int32_t)std::exp(uniform() * std::log(most + 1.0));
}
static int coin(int n) { return (int)(uniform() * n); }
static void* const fake = reinterpret_cast<void*>(0x7f0000001000);
static const double CARD = 288e9;
static long accepted = 0, refused = 0;
// what a launch can be: fewer than 2^32 threads along each axis, 65535 workgroups along y and z
static void look(int rc, const char* what, long a, long b, long c, long d, int io, unsigned flags)
{
    bool good = rc == SS_OK || launches.empty();
    for (const Launch& l : launches) {
        good = good && (uint64_t)l.grid.x * l.block.x < (1ull << 32) && l.grid.x <= 0x7fffffffu && l.grid.x >= 1;
        good = good && l.grid.y >= 1 && l.grid.y <= 65535 && l.grid.z >= 1 && l.grid.z <= 65535 && l.block.x <= 1024;
    }
    if (!good) {
        std::printf("%s %ld %ld %ld %ld io %d flags %u: result %d", what, a, b, c, d, io, flags, rc);
        for (const Launch& l : launches) std::printf(", (%u %u %u) x %u", l.grid.x, l.grid.y, l.grid.z, l.block.x);
        std::printf("\n");
        std::exit(1);
    }
    rc == SS_OK ? ++accepted : ++refused;
    launches.clear();
}
"""

TAIL = r"""
int main()
{
    for (long i = 0; i < 200000; ++i) one();
    std::printf("%ld accepted, %ld refused\n", accepted, refused);
    return accepted < 20000;
}
"""


def run(tmp_path, source, body):
    src, obj, exe = (str(tmp_path / n) for n in ("launches.hip", "launches.o", "launches"))
    with open(src, "w") as f:
        f.write(HEAD.replace("SOURCE", source) + body + TAIL)
    subprocess.run([build._hipcc(), "--offload-arch=gfx950", "-std=c++17", "-O1", "-fPIC", "--offload-host-only", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), "-c", src, "-o", obj], check=True, capture_output=True)
    subprocess.run(["g++", obj, "-o", exe], check=True, capture_output=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


LINEAR = r"""
static void one()
{
    ss_qlinear_params p{};
    p.flags = (uint32_t)coin(16);
    p.io_dtype = coin(2);
    p.dim = any(131072);
    p.features = any(2147418111);
    p.batch = coin(2) ? any(65535) : any(4);
    p.seqlen = any(2147418110);
    // the tensors have to fit the card
    const double pitch = (double)ss_quant_pitch(p.dim), rows = (double)p.batch * p.seqlen, e = p.io_dtype == SS_BF16 ? 2 : 4;
    if (rows * p.features * e + p.features * pitch + rows * pitch > CARD) return;
    p.x = p.weight = p.out = p.scratch = fake;
    p.x_scale = p.scale = p.bias = static_cast<float*>(fake);
    p.scratch_bytes = ss_qlinear_scratch_bytes(&p);
    const int rc = ss_qlinear(&p, nullptr);
    look(rc, "ss_qlinear", p.batch, p.seqlen, p.dim, p.features, p.io_dtype, p.flags);
}
"""


def test_products(tmp_path):
    run(tmp_path, "ss_quant.hip", LINEAR)


def test_rows_in_8_bits(tmp_path):
    run(tmp_path, "ss_quant.hip", r"""
static void one()
{
    ss_quant_params p{};
    p.flags = (uint32_t)coin(2);
    p.io_dtype = coin(2);
    p.dim = any(131072);
    p.batch = coin(2) ? any(65535) : any(4);
    p.seqlen = any(2147418110);
    const double pitch = (double)ss_quant_pitch(p.dim), rows = (double)p.batch * p.seqlen;
    if (rows * p.dim * (p.io_dtype == SS_BF16 ? 2 : 4) + rows * pitch > CARD) return;
    p.x = p.q = p.scratch = fake;
    p.scale = static_cast<float*>(fake);
    p.scratch_bytes = ss_quant_rows_scratch_bytes(&p);
    look(ss_quant_rows(&p, nullptr), "ss_quant_rows", p.batch, p.seqlen, p.dim, 0, p.io_dtype, p.flags);
}
""")


GATE = r"""
static void one()
{
    ss_gate_bwd_params q{};
    ss_gate_params& p = q.fwd;
    p.io_dtype = coin(2);
    p.flags = (uint32_t)coin(256);
    p.batch = coin(2) ? 1 : any(1 << 24);
    p.dim = any(2147483646);
    p.seqlen = coin(8) ? any(1 << 22) : any(2147481599);
    if (uniform() < 0.05) {   // rows about the most threads that teams of four waves have, lengths whose pieces fill them
        p.batch = 1 + coin(2);
        p.dim = ((1 << 24) - 300 + coin(600)) / p.batch;
        p.seqlen = 1500 + coin(600);
    }
    const double one_tensor = (double)p.batch * p.dim * p.seqlen * (p.io_dtype == SS_BF16 ? 2 : 4);
    if (2 * one_tensor > CARD) return;   // one tensor may serve as several inputs
    p.x = p.f = p.i = p.z = p.out = p.workspace = fake;
    p.x_batch = p.f_batch = p.i_batch = p.z_batch = (int64_t)p.dim * p.seqlen;
    p.rate = p.f_bias = p.i_bias = p.h0 = p.h_last = static_cast<float*>(fake);
    p.reset = static_cast<uint8_t*>(fake);
    p.workspace_bytes = ss_gate_workspace_bytes(&p, 1);
    const bool forward = ss_gate_fwd(&p, nullptr) == SS_OK;
    look(forward ? SS_OK : SS_ERR_UNSUPPORTED, "ss_gate_fwd", p.batch, p.dim, p.seqlen, 0, p.io_dtype, p.flags);
    if (5 * one_tensor > CARD) return;
    q.dout = q.dx = q.df = q.di = q.dz = fake;
    q.dh_last = q.drate = q.df_bias = q.di_bias = q.dh0 = static_cast<float*>(fake);
    q.dx_batch = q.df_batch = q.di_batch = q.dz_batch = (int64_t)p.dim * p.seqlen;
    const bool backward = ss_gate_bwd(&q, nullptr) == SS_OK;
    look(backward == forward ? (backward ? SS_OK : SS_ERR_UNSUPPORTED) : 1, "ss_gate_bwd", p.batch, p.dim, p.seqlen, 0, p.io_dtype, p.flags);
    ss_gate_step_params t{};
    t.batch = p.batch; t.dim = p.dim; t.io_dtype = p.io_dtype;
    t.flags = p.flags & (SS_GATE_HAS_I | SS_GATE_HAS_Z);
    t.x_t = t.f_t = t.i_t = t.z_t = t.out_t = fake;
    t.x_batch = t.f_batch = t.i_batch = t.z_batch = p.dim;
    t.h = static_cast<float*>(fake); t.rate = p.rate;
    look(ss_gate_step(&t, nullptr), "ss_gate_step", p.batch, p.dim, 1, 0, p.io_dtype, t.flags);
}
"""


def test_recurrence(tmp_path):
    run(tmp_path, "ss_gate.hip", GATE)


NORM = r"""
static void one()
{
    ss_norm_bwd_params q{};
    ss_norm_params& p = q.fwd;
    p.io_dtype = coin(2);
    p.flags = (uint32_t)coin(16) | SS_NORM_SAVE_STATS;
    p.rows = any(2147418111);
    p.width = any(2147418111);
    p.eps = 1e-5f;
    const double io = (double)p.rows * p.width * (p.io_dtype == SS_BF16 ? 2 : 4);
    const bool res = p.flags & SS_NORM_HAS_RESIDUAL;
    if ((res ? 3 : 1) * io > CARD) return;   // out may be x, summed the residual
    p.x = p.residual = p.out = p.summed = fake;
    p.weight = p.bias = p.stats = static_cast<float*>(fake);
    look(ss_norm_fwd(&p, nullptr), "ss_norm_fwd", p.rows, p.width, 0, 0, p.io_dtype, p.flags);
    if (3 * io > CARD) return;
    q.dout = q.dsummed = q.dx = q.dresidual = q.workspace = fake;
    q.dweight = q.dbias = static_cast<float*>(fake);
    q.workspace_bytes = ss_norm_workspace_bytes(&p);
    look(ss_norm_bwd(&q, nullptr), "ss_norm_bwd", p.rows, p.width, 0, 0, p.io_dtype, p.flags);
}
"""


def test_norm(tmp_path):
    run(tmp_path, "ss_norm.hip", NORM)
