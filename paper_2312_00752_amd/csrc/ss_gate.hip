// Gated linear recurrence for gfx950: forward, backward and single-token step, with their C-ABI
// entry points (see include/ss_gate.h).
//
// Per element the operation reads two to four values, writes one (backward: as many gradients as inputs) and evaluates six to
// eight transcendental functions; the recurrence itself is two multiply-adds.  Unlike the selective scan it has one state
// per row, so a lane cannot walk a row: a wave does, in pieces.
//
// A lane owns 8 consecutive steps (a slice: 16 bytes of bf16), G lanes own a piece of 8 G steps of one row, and a wave has
// 64 / G rows.  With every step an affine map h -> a h + b, a lane composes its slice's maps into one (A, B), the lanes'
// maps are composed by a prefix scan in registers (DPP within rows of 16 lanes, the four row totals through scalar
// registers), and with the state that stands before its slice known each lane walks the slice once more.  The expanded
// a, b and h live in registers only.  The backward pass recomputes the states of a piece from the state
// before it, which the forward pass left (one float per piece), and runs the adjoint through the same scan backwards in time:
//
//     lam_t = dy_t + G_{t+1},   G_t = a_t lam_t,   dL/d(log a_t) = lam_t a_t (h_{t-1} - g_t x_t a_t / m_t)
//
// G_t is again an affine map of G_{t+1}, with a_t and b = a_t dy_t.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>

#include "ss_gate.h"
#include "ss_slices.h"

namespace ss {

constexpr int LANE_STEPS = 8;                       // steps of one lane
constexpr int GATE_PIECE = WAVE * LANE_STEPS;       // steps of a whole wave: the distance of the checkpoints
constexpr int GATE_WAVES = 4;                  // waves of a workgroup where each has rows of its own
constexpr float GATE_LOG2E = 1.44269504088896340736f;
// 2^-126, the least normal number: of anything smaller the hardware's square root is 0 and its reciprocal square root infinite, so a step
// whose 1 - a^2 lies below it has m = 0 in every pass, and no derivative of m
constexpr float GATE_LEAST_M2 = 0x1p-126f;

struct GateArgs {
    int B, D, L, R;                            // R = B D rows
    int pieces, nseg, spp;                     // pieces of GATE_PIECE steps; segments and their pieces
    int nmap, ppm;                             // maps that the segments are composed of, and their pieces
    unsigned flags;
    const void *x, *f, *i, *z;
    int64_t xb, fb, ib, zb;
    const float *rate, *f_bias, *i_bias, *h0;
    const uint8_t* reset;
    void* out;
    float* h_last;
    float* ckpt;                               // (pieces, R): the state before each piece; or null
    float2* agg;                               // (R, nmap): the composed maps of ppm pieces each
    float* carry;                              // (nseg, R): the state (backward: G) that enters a segment; null for one segment
    const void* dout;
    const float* dh_last;
    void *dx, *df, *di, *dz;
    int64_t dxb, dfb, dib, dzb;
    float *part_rate, *part_f, *part_i;        // (nseg, R) sums of a row's segment
    float* dh0;
};

// ---- affine maps ------------------------------------------------------------------------
// h -> A h + B.  With resets, A < 0 says that a reset lies within: the map is then the constant B whatever came before,
// also where that is not finite (A is never negative otherwise, and a product with 0 would let NaN through).
template <bool RST>
__device__ __forceinline__ void affine_after(float& A, float& B, float A0, float B0)   // (A, B) after (A0, B0)
{
    if constexpr (RST) {
        const bool own = A < 0.0f;
        B = own ? B : fmaf(A, B0, B);
        A = own || A0 < 0.0f ? -1.0f : A * A0;
    } else {
        B = fmaf(A, B0, B);
        A *= A0;
    }
}
template <bool RST>
__device__ __forceinline__ float affine_of(float A, float B, float h)
{
    if constexpr (RST) return A < 0.0f ? B : fmaf(A, h, B);
    else return fmaf(A, h, B);
}

template <int CTRL>
__device__ __forceinline__ float dpp_or(float v, float other)   // v of the lane that CTRL names, `other` where there is none in the row
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(other), (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }

template <int G, bool BACK, bool RST, int K>
__device__ __forceinline__ void scan_step(float& A, float& B, int gl)
{
    if constexpr (K < G && K < 16) {
        constexpr int CTRL = (BACK ? 0x100 : 0x110) + K;   // row_shl / row_shr
        float A0 = dpp_or<CTRL>(A, 1.0f), B0 = dpp_or<CTRL>(B, 0.0f);
        if constexpr (G < 16) {   // groups end inside a row
            const bool have = BACK ? gl + K < G : gl >= K;
            A0 = have ? A0 : 1.0f;
            B0 = have ? B0 : 0.0f;
        }
        affine_after<RST>(A, B, A0, B0);
    }
}
// (A, B): a lane's slice as one map.  scan() composes those of the lanes before it (BACK: behind it, in time) onto it; apply() returns
// the state before the slice, given `c`, the one before the piece, which becomes the one after it.
template <int G, bool BACK>
struct LaneScan {
    float A, B;                  // through the lane, within its row of 16 lanes (its group, if smaller)
    float rA[4], rB[4];          // G == 64: the rows of lanes, in time's order
    template <bool RST>
    __device__ __forceinline__ void scan(float A_, float B_, int lane)
    {
        A = A_;
        B = B_;
        const int gl = lane & (G - 1);
        scan_step<G, BACK, RST, 1>(A, B, gl);
        scan_step<G, BACK, RST, 2>(A, B, gl);
        scan_step<G, BACK, RST, 4>(A, B, gl);
        scan_step<G, BACK, RST, 8>(A, B, gl);
        if constexpr (G == WAVE) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                rA[r] = lane_value(A, BACK ? 48 - 16 * r : 15 + 16 * r);
                rB[r] = lane_value(B, BACK ? 48 - 16 * r : 15 + 16 * r);
            }
        }
    }
    template <bool RST>
    __device__ __forceinline__ void whole(float& WA, float& WB) const   // the wave's map
    {
        WA = rA[0];
        WB = rB[0];
#pragma unroll
        for (int r = 1; r < 4; ++r) {
            float A1 = rA[r], B1 = rB[r];
            affine_after<RST>(A1, B1, WA, WB);
            WA = A1;
            WB = B1;
        }
    }
    template <bool RST>
    __device__ __forceinline__ float apply(float& c, int lane) const
    {
        const int gl = lane & (G - 1);
        constexpr int CTRL = BACK ? 0x101 : 0x111;
        float Ae = dpp_or<CTRL>(A, 1.0f), Be = dpp_or<CTRL>(B, 0.0f);
        float cin = c;
        if constexpr (G == WAVE) {
            const float c0 = c, c1 = affine_of<RST>(rA[0], rB[0], c0), c2 = affine_of<RST>(rA[1], rB[1], c1), c3 = affine_of<RST>(rA[2], rB[2], c2);
            c = affine_of<RST>(rA[3], rB[3], c3);
            const int row = BACK ? 3 - (lane >> 4) : lane >> 4;
            cin = row < 2 ? (row == 0 ? c0 : c1) : (row == 2 ? c2 : c3);
        } else {
            if constexpr (G < 16) {
                const bool first = gl == (BACK ? G - 1 : 0);
                Ae = first ? 1.0f : Ae;
                Be = first ? 0.0f : Be;
            }
            c = affine_of<RST>(A, B, c);   // valid in the group's last lane (BACK: first)
        }
        return affine_of<RST>(Ae, Be, cin);
    }
};

// TEAM waves work on neighbouring pieces of one row at a time: from their pieces' maps and the state `c` before all of them each
// gets the state before its own; c becomes the one behind all.  The two halves of LDS are used in turn, so one barrier a time.
template <int TEAM, bool BACK, bool RST>
struct TeamScan {
    float2 (*lds)[TEAM];
    int turn = 0;
    __device__ __forceinline__ float operator()(float A, float B, float& c, int wave, int lane)
    {
        const int pos = BACK ? TEAM - 1 - wave : wave;
        if (lane == 0) lds[turn][pos] = make_float2(A, B);
        __syncthreads();
        const float2 m = lds[turn][lane & (TEAM - 1)];
        turn ^= 1;
        float A1 = m.x, B1 = m.y;   // lanes of a row of 16: the maps in time's order
        const int gl = lane & (TEAM - 1);
        scan_step<TEAM, false, RST, 1>(A1, B1, gl);
        scan_step<TEAM, false, RST, 2>(A1, B1, gl);
        scan_step<TEAM, false, RST, 4>(A1, B1, gl);
        scan_step<TEAM, false, RST, 8>(A1, B1, gl);
        const float h = affine_of<RST>(A1, B1, c);
        const float before = pos == 0 ? c : lane_value(h, pos - 1);
        c = lane_value(h, TEAM - 1);
        return before;
    }
};

// ---- reset marks ---------------------------------------------------------------------------
// Eight reset marks, asked for like a slice (nothing waits between the request and the use) and shifted into place when they are
// used, zeros past the row.
template <bool TINY>
__device__ __forceinline__ uint2 marks_request(const uint8_t* row, int t0, int L)
{
    if constexpr (TINY)
        if (L < 8) {
            uint32_t w[2] = {0u, 0u};
            for (int j = 0; j < 8; ++j)
                if (t0 + j < L) w[j >> 2] |= uint32_t(row[t0 + j]) << (8 * (j & 3));
            return make_uint2(w[0], w[1]);
        }
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    const u2 v = load_any<u2>(row + min(t0, L - 8), 0u);
    return make_uint2(v[0], v[1]);
}
__host__ __device__ __forceinline__ uint2 marks_settle(uint2 m, int t0, int L)
{
    const int past = t0 - (L - 8);   // L < 8: the marks are in place
    if (past <= 0 || L < 8) return m;
    const uint64_t w = past < 8 ? ((uint64_t(m.y) << 32) | m.x) >> (8 * past) : 0;
    return make_uint2((uint32_t)w, (uint32_t)(w >> 32));
}
__device__ __forceinline__ bool marked(uint2 m, int j) { return ((j < 4 ? m.x : m.y) & (0xffu << (8 * (j & 3)))) != 0; }

// ---- the gates of one step ------------------------------------------------------------------
// sigmoid by the hardware's exponential and reciprocal (1 ulp each).  The exponential's argument is rounded, so the relative error grows
// with |v|: at most (1.25 |v| + 6) 2^-24, 1e-6 at -8 and 7e-6 at -87; below -87.33, where it is less than 2^-126, it becomes 0.
__device__ __forceinline__ float gate_sigmoid(float v) { return rcp_fast(1.0f + exp2_fast(-GATE_LOG2E * v)); }
// 1 - a^2 with a = exp(-y / 2): the difference loses 2^-24 / y, so below y = 1/8 the series y (1 - y/2 + y^2/6 - ...), whose
// first term left out is y^5 / 720 (4e-8); the difference is off by 1e-6 there and less above.
__device__ __forceinline__ float one_minus_square(float y, float a)
{
    const float p = y * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.0f / 120.0f, -1.0f / 24.0f), 1.0f / 6.0f), -0.5f), 1.0f);
    return y < 0.125f ? p : fmaf(-a, a, 1.0f);
}

struct Channel {
    float rate, f_bias, i_bias;
};
__device__ __forceinline__ Channel channel_of(const GateArgs& a, int d)
{
    Channel c;
    c.rate = a.rate[d];
    c.f_bias = (a.flags & SS_GATE_HAS_F_BIAS) ? a.f_bias[d] : 0.0f;
    c.i_bias = (a.flags & SS_GATE_HAS_I_BIAS) ? a.i_bias[d] : 0.0f;
    return c;
}

// Where a lane works: its row, and what is common to the row's slices.
template <int G, int TEAM>
struct Place {
    int lane, gl, row, b, d, limit;   // limit: slice_limit of the row
    int member;                      // of the team
    bool valid, whole;
    __device__ __forceinline__ Place(const GateArgs& a)
    {
        lane = threadIdx.x & (WAVE - 1);
        gl = lane & (G - 1);
        member = TEAM > 1 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x / WAVE)) : 0;
        const int wave = TEAM > 1 ? (int)blockIdx.x : (int)blockIdx.x * GATE_WAVES + (int)(threadIdx.x / WAVE);
        row = wave * (WAVE / G) + lane / G;
        if constexpr (G == WAVE) row = __builtin_amdgcn_readfirstlane(row);
        valid = row < a.R;
        row = min(row, a.R - 1);
        b = row / a.D;
        d = row - b * a.D;
        whole = slice_whole(a.L, (wave + 1) * (WAVE / G) >= a.R);   // the tensor's last row is in the last wave only
        limit = slice_limit(a.L, whole);
    }
    template <typename T>
    __device__ __forceinline__ const T* in(const void* p, int64_t batch, int L) const { return static_cast<const T*>(p) + b * batch + (int64_t)d * L; }
    template <typename T>
    __device__ __forceinline__ typename io8<T>::raw request(const T* row, int t0, int L) const { return slice_request<T, G == 4>(row, t0, L, limit); }
    template <typename T>
    __device__ __forceinline__ void settle(typename io8<T>::raw& r, int t0, int L) const { slice_settle<T>(r, t0, L, limit, whole); }
    template <typename T>
    __device__ __forceinline__ T* to(void* p, int64_t batch, int L) const { return static_cast<T*>(p) + b * batch + (int64_t)d * L; }
};

// ---- forward ---------------------------------------------------------------------------------
template <typename T, bool HI>
struct fwd_raw {
    typename io8<T>::raw x, f, i;
    uint2 m;
};
// a and b of the slice's steps; steps past the row leave the state as it is.
template <typename T, bool HI, bool RST>
__device__ __forceinline__ void steps_of(const fwd_raw<T, HI>& r, const Channel& c, int n, float (&av)[8], float (&bv)[8])
{
    float x[8], f[8], iv[8];
    io8<T>::unpack(r.x, x);
    io8<T>::unpack(r.f, f);
    if constexpr (HI) io8<T>::unpack(r.i, iv);
    const float k = -GATE_LOG2E * c.rate, rate2 = 2.0f * c.rate;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float s = gate_sigmoid(f[j] + c.f_bias);
        const float a = exp2_fast(k * s);
        float m = __builtin_amdgcn_sqrtf(one_minus_square(rate2 * s, a));
        if constexpr (RST) m = marked(r.m, j) ? 1.0f : m;
        float b = m * x[j];
        if constexpr (HI) b *= gate_sigmoid(iv[j] + c.i_bias);
        av[j] = RST && marked(r.m, j) ? -1.0f : a;
        bv[j] = b;
    }
    if (n < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            av[j] = j < n ? av[j] : 1.0f;
            bv[j] = j < n ? bv[j] : 0.0f;
        }
    }
}
template <bool RST>
__device__ __forceinline__ void slice_map(const float (&av)[8], const float (&bv)[8], float& A, float& B)
{
    A = av[0];
    B = bv[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) {
        float A1 = av[j], B1 = bv[j];
        affine_after<RST>(A1, B1, A, B);
        A = A1;
        B = B1;
    }
}

template <int TEAM> constexpr int gate_threads() { return (TEAM > 1 ? TEAM : GATE_WAVES) * WAVE; }

// Bound by HBM on full grids: 32768 rows of 2048 bf16 with input gate and z (671 MB) 145 us, 4.6 TB/s; 16384 of 1531 50 us, 5.0 TB/s; 256
// rows of 2^20 float32 without z (4.3 GB) 860 us, 5.0 TB/s.  With reset marks 1536
// rows of 4097 float32 35 us, 3.6 TB/s: 4097 steps are nine pieces, three rounds of a team of four.  (Marks are selects in every step; a second path
// without them for waves that have no mark took 117 registers instead of 77, and 37 us.)
//
// AHEAD: rounds whose inputs have been requested while one is worked on.  Two where a SIMD has but one or two waves: 256 rows of 243260 float32
// 357 us with one, 268 with two, bf16 199 / 182, 384 of 100182 197 / 178 and 113 / 109; but 700 of 9000 bf16 18.3 / 20.1, 1024 of 16384 32.7 / 35.4.
template <typename T, int G, int TEAM, int AHEAD, bool HI, bool HZ, bool RST>
__global__ __launch_bounds__(gate_threads<TEAM>()) void gate_fwd_kernel(GateArgs a)
{
    const Place<G, TEAM> at(a);
    const Channel ch = channel_of(a, at.d);
    const T *x = at.template in<T>(a.x, a.xb, a.L), *f = at.template in<T>(a.f, a.fb, a.L);
    const T* iv = HI ? at.template in<T>(a.i, a.ib, a.L) : nullptr;
    const T* z = HZ ? at.template in<T>(a.z, a.zb, a.L) : nullptr;
    T* out = static_cast<T*>(a.out) + (int64_t)at.row * a.L;
    const uint8_t* reset = RST ? a.reset + (int64_t)at.b * a.L : nullptr;
    const int seg = blockIdx.y, p0 = seg * a.spp, p1 = min(p0 + a.spp, a.pieces);
    float c = 0.0f;   // the state before what the team has at hand
    if (a.nseg > 1) c = a.carry[(int64_t)seg * a.R + at.row];   // the first segment's too: h_last, which the last one writes, may be h0
    else if (a.flags & SS_GATE_HAS_H0) c = a.h0[at.row];
    __shared__ float2 maps[2][TEAM];
    TeamScan<TEAM, false, RST> team{maps};

    struct Request {
        fwd_raw<T, HI> r;
        typename io8<T>::raw rz;
    };
    Request req[AHEAD];
    auto load = [&](int p, Request& to) {
        auto& r = to.r;
        auto& rz = to.rz;
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS;
        r.x = at.template request<T>(x, t0, a.L);
        r.f = at.template request<T>(f, t0, a.L);
        if constexpr (HI) r.i = at.template request<T>(iv, t0, a.L);
        if constexpr (HZ) rz = at.template request<T>(z, t0, a.L);
        if constexpr (RST) r.m = marks_request<G == 4>(reset, t0, a.L);
    };
    // a team's members that have no piece left take part with maps that change nothing
    auto round = [&](int q, Request& now) {
        auto& r = now.r;
        auto& rz = now.rz;
        const int p = q + at.member, t0 = p * GATE_PIECE + at.gl * LANE_STEPS, n = p < p1 ? a.L - t0 : 0;
        float av[8], bv[8], zv[8], y[8];
        if (!at.whole) {
            at.template settle<T>(r.x, t0, a.L);
            at.template settle<T>(r.f, t0, a.L);
            if constexpr (HI) at.template settle<T>(r.i, t0, a.L);
            if constexpr (HZ) at.template settle<T>(rz, t0, a.L);
        }
        if constexpr (RST) r.m = marks_settle(r.m, t0, a.L);
        LaneScan<G, false> lanes;
        float A, B;
        steps_of<T, HI, RST>(r, ch, n, av, bv);
        if constexpr (HZ) io8<T>::unpack(rz, zv);
        if (q + AHEAD * TEAM < p1) load(min(p + AHEAD * TEAM, a.pieces - 1), now);
        slice_map<RST>(av, bv, A, B);
        lanes.template scan<RST>(A, B, at.lane);
        if constexpr (TEAM > 1) lanes.template whole<RST>(A, B);
        float own = c;
        if constexpr (TEAM > 1) own = team(A, B, c, at.member, at.lane);
        if (a.ckpt && at.valid && at.gl == 0 && p < p1) a.ckpt[(int64_t)p * a.R + at.row] = own;
        float h = lanes.template apply<RST>(own, at.lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h = affine_of<RST>(av[j], bv[j], h);
            y[j] = HZ ? h * zv[j] * gate_sigmoid(zv[j]) : h;
        }
        if constexpr (TEAM == 1) c = own;
        if (at.valid) slice_store<T>(out, t0, n, y);
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (k == 0 || p0 + k * TEAM < p1) load(min(p0 + k * TEAM + at.member, a.pieces - 1), req[k]);
    for (int q = p0; q < p1; q += AHEAD * TEAM) {
        round(q, req[0]);
        if constexpr (AHEAD == 2) {
            if (q + TEAM >= p1) break;
            round(q + TEAM, req[1]);
        }
    }
    if (a.h_last && at.valid && seg == a.nseg - 1 && at.member == 0 && at.gl == (G == WAVE ? 0 : G - 1)) a.h_last[at.row] = c;
}

// ppm pieces as one map: one wave each (a segment is a whole number of them).  64 rows of 2^20 bf16, no input gate (268 MB), 77 us.
template <typename T, bool HI, bool RST>
__global__ __launch_bounds__(GATE_WAVES* WAVE) void gate_fwd_map_kernel(GateArgs a)
{
    const Place<WAVE, 1> at(a);
    const Channel ch = channel_of(a, at.d);
    const T *x = at.template in<T>(a.x, a.xb, a.L), *f = at.template in<T>(a.f, a.fb, a.L);
    const T* iv = HI ? at.template in<T>(a.i, a.ib, a.L) : nullptr;
    const uint8_t* reset = RST ? a.reset + (int64_t)at.b * a.L : nullptr;
    const int map = blockIdx.y, p0 = map * a.ppm, p1 = min(p0 + a.ppm, a.pieces);
    fwd_raw<T, HI> r;
    auto load = [&](int p) {
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS;
        r.x = at.template request<T>(x, t0, a.L);
        r.f = at.template request<T>(f, t0, a.L);
        if constexpr (HI) r.i = at.template request<T>(iv, t0, a.L);
        if constexpr (RST) r.m = marks_request<false>(reset, t0, a.L);
    };
    float sA = 1.0f, sB = 0.0f;
    load(p0);
    for (int p = p0; p < p1; ++p) {
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS;
        if (!at.whole) {
            at.template settle<T>(r.x, t0, a.L);
            at.template settle<T>(r.f, t0, a.L);
            if constexpr (HI) at.template settle<T>(r.i, t0, a.L);
        }
        if constexpr (RST) r.m = marks_settle(r.m, t0, a.L);
        float av[8], bv[8], A, B;
        steps_of<T, HI, RST>(r, ch, a.L - t0, av, bv);
        if (p + 1 < p1) load(p + 1);
        slice_map<RST>(av, bv, A, B);
        LaneScan<WAVE, false> lanes;
        lanes.template scan<RST>(A, B, at.lane);
        lanes.template whole<RST>(A, B);
        affine_after<RST>(A, B, sA, sB);
        sA = A;
        sB = B;
    }
    if (at.valid && at.lane == 0) a.agg[(int64_t)at.row * a.nmap + map] = make_float2(sA, sB);
}

// The state that enters each segment, from the maps: a wave a row, whose lanes have neighbouring segments; BACK: the adjoint, from the
// last segment on.  per: maps of a segment.
template <bool RST, bool BACK>
__global__ __launch_bounds__(WAVE) void gate_carry_kernel(GateArgs a)
{
    const int row = blockIdx.x, lane = threadIdx.x, per = a.spp / a.ppm, share = (a.nseg + WAVE - 1) / WAVE;
    const float2* const maps = a.agg + (int64_t)row * a.nmap;
    float c = 0.0f;
    if (BACK) { if (a.dh_last) c = a.dh_last[row]; }
    else if (a.flags & SS_GATE_HAS_H0) c = a.h0[row];
    // the lane's segments in time's order (BACK: against it) from s0 on
    const int s0 = lane * share, s1 = min(s0 + share, a.nseg);
    auto segment = [&](int s, float& A, float& B) {   // composed onto (A, B)
        const int first = (BACK ? a.nseg - 1 - s : s) * per;
        for (int k = 0; k < per; ++k) {
            const int m = first + (BACK ? per - 1 - k : k);
            if (m >= a.nmap) continue;
            float2 v = maps[m];
            affine_after<RST>(v.x, v.y, A, B);
            A = v.x;
            B = v.y;
        }
    };
    float A = 1.0f, B = 0.0f;
    for (int s = s0; s < s1; ++s) segment(s, A, B);
    LaneScan<WAVE, false> lanes;
    lanes.template scan<RST>(A, B, lane);
    float h = lanes.template apply<RST>(c, lane);
    for (int s = s0; s < s1; ++s) {
        a.carry[(int64_t)(BACK ? a.nseg - 1 - s : s) * a.R + row] = h;
        A = 1.0f;
        B = 0.0f;
        segment(s, A, B);
        h = affine_of<RST>(A, B, h);
    }
}

// ---- backward --------------------------------------------------------------------------------
// With lam_t the gradient that reaches h_t, v = m g x the step's input and m' = dm / d(log a) = -a^2 / m:
//     dx = lam m g,   di = lam v (1 - g),   d(log a) = lam (a h_{t-1} - (g x) a^2 / m) = lam a (h_{t-1} - g x a / m)
//     log a = -rate s:   df = -d(log a) rate s (1 - s),   drate = -sum d(log a) s
//     dz = dout h (sz + z sz (1 - sz)),   dy = dout z sz
//
// Bound by HBM as well: 32768 rows of 2048 bf16 with input gate and z (1.2 GB) 226 us, 5.3 TB/s; 256 rows of 2^20 float32 without z (7.5 GB) 1520
// us, 4.9 TB/s; with marks 1536 rows of 4097 float32 51 us, 4.4 TB/s (two paths: 176 registers, two waves a SIMD instead of three, 57).
template <typename T, int G, int TEAM, bool HI, bool HZ, bool RST>
__global__ __launch_bounds__(gate_threads<TEAM>()) void gate_bwd_kernel(GateArgs a)
{
    const Place<G, TEAM> at(a);
    const Channel ch = channel_of(a, at.d);
    const T *x = at.template in<T>(a.x, a.xb, a.L), *f = at.template in<T>(a.f, a.fb, a.L);
    const T* iv = HI ? at.template in<T>(a.i, a.ib, a.L) : nullptr;
    const T* z = HZ ? at.template in<T>(a.z, a.zb, a.L) : nullptr;
    const T* dout = static_cast<const T*>(a.dout) + (int64_t)at.row * a.L;
    T *dx = at.template to<T>(a.dx, a.dxb, a.L), *df = at.template to<T>(a.df, a.dfb, a.L);
    T* di = HI ? at.template to<T>(a.di, a.dib, a.L) : nullptr;
    T* dz = HZ ? at.template to<T>(a.dz, a.dzb, a.L) : nullptr;
    const uint8_t* reset = RST ? a.reset + (int64_t)at.b * a.L : nullptr;
    const int seg = blockIdx.y, p0 = seg * a.spp, p1 = min(p0 + a.spp, a.pieces);
    float c = 0.0f;   // G behind the piece
    if (a.nseg > 1) c = a.carry[(int64_t)seg * a.R + at.row];   // the last segment's too: dh0, which the first one writes, may be dh_last
    else if (a.dh_last) c = a.dh_last[at.row];
    const float k = -GATE_LOG2E * ch.rate, rate2 = 2.0f * ch.rate;
    float sum_q = 0.0f, sum_f = 0.0f, sum_i = 0.0f;
    __shared__ float2 maps[2][TEAM];
    TeamScan<TEAM, true, RST> team{maps};

    fwd_raw<T, HI> r;
    typename io8<T>::raw rz, rd;
    auto load = [&](int p) {
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS;
        r.x = at.template request<T>(x, t0, a.L);
        r.f = at.template request<T>(f, t0, a.L);
        rd = at.template request<T>(dout, t0, a.L);
        if constexpr (HI) r.i = at.template request<T>(iv, t0, a.L);
        if constexpr (HZ) rz = at.template request<T>(z, t0, a.L);
        if constexpr (RST) r.m = marks_request<G == 4>(reset, t0, a.L);
    };
    // the team's pieces from the last ones on, the first time as many as are left over
    const int top = p0 + (p1 - 1 - p0) / TEAM * TEAM;
    load(min(top + at.member, a.pieces - 1));
    for (int q = top; q >= p0; q -= TEAM) {
        const int p = q + at.member, t0 = p * GATE_PIECE + at.gl * LANE_STEPS, n = p < p1 ? a.L - t0 : 0;
        float start = a.ckpt[(int64_t)min(p, a.pieces - 1) * a.R + at.row];
        float av[8], bv[8], sv[8], gx[8], gv[8], iq[8], hp[8], dy[8], o[8], zv[8];   // iq: 1 / m
        const uint2 marks = RST ? marks_settle(r.m, t0, a.L) : r.m;
        if (!at.whole) {
            at.template settle<T>(r.x, t0, a.L);
            at.template settle<T>(r.f, t0, a.L);
            at.template settle<T>(rd, t0, a.L);
            if constexpr (HI) at.template settle<T>(r.i, t0, a.L);
            if constexpr (HZ) at.template settle<T>(rz, t0, a.L);
        }
        LaneScan<G, true> back;
        float A, B;
        {
            float xv[8], fv[8], ivv[8];
            io8<T>::unpack(r.x, xv);
            io8<T>::unpack(r.f, fv);
            io8<T>::unpack(rd, dy);
            if constexpr (HI) io8<T>::unpack(r.i, ivv);
            if constexpr (HZ) io8<T>::unpack(rz, zv);
            if (q > p0) load(p - TEAM);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = j < n, mk = RST && marked(marks, j);
                const float s = gate_sigmoid(fv[j] + ch.f_bias);
                const float aa = exp2_fast(k * s);
                const float m2 = one_minus_square(rate2 * s, aa);
                float rm = __builtin_amdgcn_rsqf(m2);
                rm = m2 < GATE_LEAST_M2 ? 0.0f : rm;
                const float g = HI ? gate_sigmoid(ivv[j] + ch.i_bias) : 1.0f;
                const float m = mk ? 1.0f : m2 * rm;
                sv[j] = s;
                gv[j] = g;
                iq[j] = rm;
                gx[j] = in ? g * xv[j] : 0.0f;
                av[j] = in ? (mk ? -1.0f : aa) : 1.0f;
                bv[j] = in ? m * gx[j] : 0.0f;
                dy[j] = in ? dy[j] : 0.0f;
            }
        }
        slice_map<RST>(av, bv, A, B);
        LaneScan<G, false> lanes;
        lanes.template scan<RST>(A, B, at.lane);
        float h = lanes.template apply<RST>(start, at.lane);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            hp[j] = h;
            h = affine_of<RST>(av[j], bv[j], h);
            if constexpr (HZ) {
                const float sz = gate_sigmoid(zv[j]);
                o[j] = dy[j] * h * fmaf(zv[j] * sz, 1.0f - sz, sz);
                dy[j] = j < n ? dy[j] * zv[j] * sz : 0.0f;
            }
        }
        // G of the slice as one map, from its last step to its first: G_t = a (dy + G_{t+1}), 0 at a reset
        A = 1.0f;
        B = 0.0f;
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            float A1 = av[j], B1 = av[j] * dy[j];
            if (RST && A1 < 0.0f) B1 = 0.0f;
            affine_after<RST>(A1, B1, A, B);
            A = A1;
            B = B1;
        }
        back.template scan<RST>(A, B, at.lane);
        if constexpr (TEAM > 1) back.template whole<RST>(A, B);
        if constexpr (HZ)
            if (at.valid) slice_store<T>(dz, t0, n, o);
        float own = c;
        if constexpr (TEAM > 1) own = team(A, B, c, at.member, at.lane);
        float sq = 0.0f, sf = 0.0f, si = 0.0f;
        float gz[8], o2[8];
        float gn = back.template apply<RST>(own, at.lane);
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            const bool in = j < n, mk = RST && av[j] < 0.0f;
            const float lam = dy[j] + gn;
            const float m = mk ? 1.0f : (iq[j] == 0.0f ? 0.0f : rcp_fast(iq[j]));
            gz[j] = lam * m * gv[j];                      // dx
            if constexpr (HI) {
                o[j] = in ? lam * bv[j] * (1.0f - gv[j]) : 0.0f;
                si += o[j];
            }
            const float dr = mk || !in ? 0.0f : lam * av[j] * (hp[j] - gx[j] * av[j] * iq[j]) * sv[j];
            sq -= dr;
            // not by way of dr = 0: sv is NaN where f is, behind the row or at a mark
            o2[j] = mk || !in ? 0.0f : -ch.rate * dr * (1.0f - sv[j]);
            sf += o2[j];
            gn = mk ? 0.0f : (in ? av[j] * lam : gn);
        }
        if constexpr (TEAM == 1) c = own;
        sum_q += sq;
        sum_f += sf;
        sum_i += si;
        if (at.valid) {
            slice_store<T>(dx, t0, n, gz);
            slice_store<T>(df, t0, n, o2);
            if constexpr (HI) slice_store<T>(di, t0, n, o);
        }
    }
    if (a.dh0 && at.valid && seg == 0 && at.member == 0 && at.gl == 0) a.dh0[at.row] = c;
#pragma unroll
    for (int s = 1; s < G; s *= 2) {
        sum_q += __shfl_xor(sum_q, s);
        sum_f += __shfl_xor(sum_f, s);
        if constexpr (HI) sum_i += __shfl_xor(sum_i, s);
    }
    if constexpr (TEAM > 1) {
        __shared__ float sums[3][TEAM];
        if (at.lane == 0) {
            sums[0][at.member] = sum_q;
            sums[1][at.member] = sum_f;
            sums[2][at.member] = sum_i;
        }
        __syncthreads();
        sum_q = sum_f = sum_i = 0.0f;
#pragma unroll
        for (int k = 0; k < TEAM; ++k) {
            sum_q += sums[0][k];
            sum_f += sums[1][k];
            sum_i += sums[2][k];
        }
    }
    if (at.valid && at.member == 0 && at.gl == 0) {
        const int64_t e = (int64_t)seg * a.R + at.row;
        a.part_rate[e] = sum_q;
        if (a.part_f) a.part_f[e] = sum_f;
        if (HI && a.part_i) a.part_i[e] = sum_i;
    }
}

// ppm pieces' adjoint as one map of G.  64 rows of 2^20 bf16 61 us.
template <typename T, bool HZ, bool RST>
__global__ __launch_bounds__(GATE_WAVES* WAVE) void gate_bwd_map_kernel(GateArgs a)
{
    const Place<WAVE, 1> at(a);
    const Channel ch = channel_of(a, at.d);
    const T* f = at.template in<T>(a.f, a.fb, a.L);
    const T* z = HZ ? at.template in<T>(a.z, a.zb, a.L) : nullptr;
    const T* dout = static_cast<const T*>(a.dout) + (int64_t)at.row * a.L;
    const uint8_t* reset = RST ? a.reset + (int64_t)at.b * a.L : nullptr;
    const int map = blockIdx.y, p0 = map * a.ppm, p1 = min(p0 + a.ppm, a.pieces);
    const float k = -GATE_LOG2E * ch.rate;
    typename io8<T>::raw rf, rd, rz;
    uint2 marks = make_uint2(0u, 0u);
    auto load = [&](int p) {
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS;
        rf = at.template request<T>(f, t0, a.L);
        rd = at.template request<T>(dout, t0, a.L);
        if constexpr (HZ) rz = at.template request<T>(z, t0, a.L);
        if constexpr (RST) marks = marks_request<false>(reset, t0, a.L);
    };
    float sA = 1.0f, sB = 0.0f;
    load(p1 - 1);
    for (int p = p1 - 1; p >= p0; --p) {
        const int t0 = p * GATE_PIECE + at.gl * LANE_STEPS, n = a.L - t0;
        if (!at.whole) {
            at.template settle<T>(rf, t0, a.L);
            at.template settle<T>(rd, t0, a.L);
            if constexpr (HZ) at.template settle<T>(rz, t0, a.L);
        }
        float fv[8], dy[8], zv[8];
        io8<T>::unpack(rf, fv);
        io8<T>::unpack(rd, dy);
        if constexpr (HZ) io8<T>::unpack(rz, zv);
        const uint2 m = marks_settle(marks, t0, a.L);
        if (p > p0) load(p - 1);
        float A = 1.0f, B = 0.0f;
#pragma unroll
        for (int j = 7; j >= 0; --j) {
            const bool in = j < n, mk = RST && marked(m, j);
            const float aa = exp2_fast(k * gate_sigmoid(fv[j] + ch.f_bias));
            const float d = HZ ? dy[j] * zv[j] * gate_sigmoid(zv[j]) : dy[j];
            float A1 = in ? (mk ? -1.0f : aa) : 1.0f, B1 = in && !mk ? aa * d : 0.0f;
            affine_after<RST>(A1, B1, A, B);
            A = A1;
            B = B1;
        }
        LaneScan<WAVE, true> lanes;
        lanes.template scan<RST>(A, B, at.lane);
        lanes.template whole<RST>(A, B);
        affine_after<RST>(A, B, sA, sB);
        sA = A;
        sB = B;
    }
    if (at.valid && at.lane == 0) a.agg[(int64_t)at.row * a.nmap + map] = make_float2(sA, sB);
}

// Sums of the rows' partial sums over batch entries and segments, in a fixed order: 16 channels of one of the three
// gradients per workgroup and round, 16 threads a channel.
__global__ __launch_bounds__(256) void gate_sums_kernel(const float* part, float* drate, float* df, float* di, int64_t plane, int D, int n)
{
    const int which = blockIdx.y;
    float* const to = which == 0 ? drate : (which == 1 ? df : di);
    if (!to) return;
    __shared__ float s[16][17];
    const int k0 = threadIdx.x >> 4;
    for (int64_t d0 = (int64_t)blockIdx.x * 16; d0 < D; d0 += (int64_t)gridDim.x * 16) {
        const int64_t d = d0 + (threadIdx.x & 15);
        float v = 0.0f;
        if (d < D)
            for (int k = k0; k < n; k += 16) v += part[which * plane + (int64_t)k * D + d];
        s[k0][threadIdx.x & 15] = v;
        __syncthreads();
        if (threadIdx.x < 16 && d < D) {
            float t = 0.0f;
            for (int k = 0; k < 16; ++k) t += s[k][threadIdx.x];
            to[d] = t;
        }
        __syncthreads();
    }
}

// seqlen == 0: state through, zero gradients
__global__ __launch_bounds__(256) void gate_fill_kernel(float* to, const float* from, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

// ---- one token -----------------------------------------------------------------------------------
// An element a thread.  64 x 4096 bf16 (4.7 MB) 3.3 us, of which a launch alone is 2.5.
template <typename T>
__global__ __launch_bounds__(256) void gate_step_kernel(ss_gate_step_params p)
{
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= p.batch * p.dim) return;
    const int b = e / p.dim, d = e - b * p.dim;
    const float s = gate_sigmoid(io_to_f32<T>(static_cast<const T*>(p.f_t)[b * p.f_batch + d]) + ((p.flags & SS_GATE_HAS_F_BIAS) ? p.f_bias[d] : 0.0f));
    const float rate = p.rate[d];
    const float a = exp2_fast(-GATE_LOG2E * rate * s);
    float m = __builtin_amdgcn_sqrtf(one_minus_square(2.0f * rate * s, a));
    const bool mk = (p.flags & SS_GATE_HAS_RESET) && p.reset_t[b];
    float v = (mk ? 1.0f : m) * io_to_f32<T>(static_cast<const T*>(p.x_t)[b * p.x_batch + d]);
    if (p.flags & SS_GATE_HAS_I)
        v *= gate_sigmoid(io_to_f32<T>(static_cast<const T*>(p.i_t)[b * p.i_batch + d]) + ((p.flags & SS_GATE_HAS_I_BIAS) ? p.i_bias[d] : 0.0f));
    const float h = mk ? v : fmaf(a, p.h[e], v);
    p.h[e] = h;
    float y = h;
    if (p.flags & SS_GATE_HAS_Z) {
        const float z = io_to_f32<T>(static_cast<const T*>(p.z_t)[b * p.z_batch + d]);
        y = h * z * gate_sigmoid(z);
    }
    static_cast<T*>(p.out_t)[e] = f32_to_io<T>(y);
}

// ---- launches --------------------------------------------------------------------------------------
template <typename F>
void with_flags(unsigned flags, F f)
{
    auto rst = [&](auto i, auto z) { (flags & SS_GATE_HAS_RESET) ? f(i, z, std::true_type{}) : f(i, z, std::false_type{}); };
    auto zz = [&](auto i) { (flags & SS_GATE_HAS_Z) ? rst(i, std::true_type{}) : rst(i, std::false_type{}); };
    (flags & SS_GATE_HAS_I) ? zz(std::true_type{}) : zz(std::false_type{});
}

// Lanes of a row: all 64 from 128 steps on; below, as many as a power of four (one piece then holds the row)
int lanes_for(int L) { return L > 16 * LANE_STEPS ? WAVE : (L > 4 * LANE_STEPS ? 16 : 4); }

template <typename T, int G, int TEAM, int AHEAD>
void launch_main(const GateArgs& a, bool bwd, hipStream_t st)
{
    const int rows = TEAM > 1 ? 1 : GATE_WAVES * (WAVE / G);
    const dim3 grid((unsigned)((a.R + rows - 1) / rows), (unsigned)a.nseg), block(gate_threads<TEAM>());
    with_flags(a.flags, [&](auto i, auto z, auto rst) {
        if (bwd) hipLaunchKernelGGL((gate_bwd_kernel<T, G, TEAM, decltype(i)::value, decltype(z)::value, decltype(rst)::value>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((gate_fwd_kernel<T, G, TEAM, AHEAD, decltype(i)::value, decltype(z)::value, decltype(rst)::value>), grid, block, 0, st, a);
    });
}
template <typename T>
void launch_all(const GateArgs& a, int team, bool bwd, hipStream_t st)
{
    if (a.nseg > 1) {
        const dim3 grid((unsigned)((a.R + GATE_WAVES - 1) / GATE_WAVES), (unsigned)a.nmap), block(GATE_WAVES * WAVE);
        with_flags(a.flags, [&](auto i, auto z, auto rst) {
            constexpr bool I = decltype(i)::value, Z = decltype(z)::value, S = decltype(rst)::value;
            if (bwd) {
                hipLaunchKernelGGL((gate_bwd_map_kernel<T, Z, S>), grid, block, 0, st, a);
                hipLaunchKernelGGL((gate_carry_kernel<S, true>), dim3((unsigned)a.R), dim3(WAVE), 0, st, a);
            } else {
                hipLaunchKernelGGL((gate_fwd_map_kernel<T, I, S>), grid, block, 0, st, a);
                hipLaunchKernelGGL((gate_carry_kernel<S, false>), dim3((unsigned)a.R), dim3(WAVE), 0, st, a);
            }
        });
    }
    const int g = lanes_for(a.L);
    if (g == 4) launch_main<T, 4, 1, 1>(a, bwd, st);
    else if (g == 16) launch_main<T, 16, 1, 1>(a, bwd, st);
    else if (team == 1) launch_main<T, WAVE, 1, 1>(a, bwd, st);
    else if (!bwd && (int64_t)a.R * a.nseg < 512) launch_main<T, WAVE, 4, 2>(a, bwd, st);
    else launch_main<T, WAVE, 4, 1>(a, bwd, st);
}

}  // namespace ss

namespace {

using ss::GateArgs;
constexpr uint32_t kGateFlags = SS_GATE_HAS_I | SS_GATE_HAS_Z | SS_GATE_HAS_F_BIAS | SS_GATE_HAS_I_BIAS | SS_GATE_HAS_RESET | SS_GATE_HAS_H0 |
                                SS_GATE_WRITE_H_LAST | SS_GATE_SAVE_FOR_BWD;
constexpr uint32_t kGateStepFlags = SS_GATE_HAS_I | SS_GATE_HAS_Z | SS_GATE_HAS_F_BIAS | SS_GATE_HAS_I_BIAS | SS_GATE_HAS_RESET;
constexpr int64_t MOST_THREADS = 0xffffffffL - 65536;   // of a launch, which has fewer than 2^32
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// How a sequence is dealt out: one wave or four share a row, and segments where the rows with their teams are still too few.
// us forward / backward with one wave / four, input gate and z, rows x steps: bf16 4096 x 1030 15.6 26.5 / 18.9 38.3, 2048 x 4096
// 22.5 34.9 / 21.0 37.8, 1024 x 16384 47.7 72.7 / 35.5 64.4, 512 x 2048 7.2 11.6 / 5.6 9.0; float32, whose requests are twice as
// wide, gains more often, and wherever the team's rounds come out even: 1536 x 4097 29.8 50.9 / 27.4 46.6, 6144 x 2048 47.5 97.9 / 41.8
// 86.8, 3000 x 2048 27.9 48.7 / 23.8 42.0, but 4096 x 1030 19.8 36.4 / 20.8 42.5.  (Teams of 8 and 16 bring up to a fifth at 256 rows and lose as much or more elsewhere.)
// In segments (two more launches and a second reading of most inputs) / whole: bf16 128 x 16384 16.0 23.1 / 12.7 21.2, 64 x 8192 12.3 16.6 / 7.5
// 12.1, 200 x 30000 29.8 43.6 / 24.4 39.2; but 128 x 65536 35.6 52.6 / 46.1 74.6, 64 x 100000 30.8 45.0 / 65.5 103.9, 1 x 1000000 19.0 25.0 / 558 944.
struct GatePlan {
    int pieces, team, nseg, spp, nmap, ppm;
};
GatePlan gate_plan(long rows, int L, int io)
{
    GatePlan g;
    g.pieces = (L + ss::GATE_PIECE - 1) / ss::GATE_PIECE;
    const bool fill = 10 * g.pieces >= 9 * ((g.pieces + 3) / 4 * 4);
    g.team = g.pieces >= 3 && (rows < (io == SS_F32 ? 2048 : 1536) || (io == SS_F32 && fill && rows <= MOST_THREADS / (4 * ss::WAVE))) ? 4 : 1;   // a team's waves are threads too
    long n = rows > 160 || g.pieces < 48 ? 1 : (768 + rows - 1) / rows;
    const long most = (g.pieces + 7) / 8;   // a segment has two rounds of its team's at least
    if (n > most) n = most;
    if (n < 1) n = 1;
    g.spp = (int)((g.pieces + n - 1) / n);
    if (n > 1) g.spp = (g.spp + g.team - 1) / g.team * g.team;
    if (g.spp < 1) g.spp = 1;
    g.nseg = g.pieces > 0 ? (g.pieces + g.spp - 1) / g.spp : 1;
    g.ppm = g.nseg > 1 ? g.spp / g.team : g.spp;   // the maps are made by single waves
    g.nmap = g.pieces > 0 ? (g.pieces + g.ppm - 1) / g.ppm : 1;
    return g;
}

// Parts of the workspace: checkpoints (pieces, R), maps (R, nmap) pairs, carries (nseg, R), and for the backward call
// the rows' sums, three planes of (nseg, R).
struct GateSpace {
    size_t ckpt, agg, carry, part, total;
};
GateSpace gate_space(long rows, const GatePlan& g, bool for_backward)
{
    GateSpace s{};
    size_t at = 0;
    const size_t one = (size_t)rows * sizeof(float);
    s.ckpt = at;
    if (for_backward) at = round_up(at + one * g.pieces, 256);
    s.agg = at;
    if (g.nseg > 1) at = round_up(at + 2 * one * g.nmap, 256);
    s.carry = at;
    if (g.nseg > 1) at = round_up(at + one * g.nseg, 256);
    s.part = at;
    if (for_backward) at = round_up(at + 3 * one * g.nseg, 256);
    s.total = at;
    return s;
}

int check_gate(const ss_gate_params* p, bool for_bwd)
{
    if (!p) return SS_ERR_NULL;
    if (p->batch < 1 || p->dim < 1 || p->seqlen < 0) return SS_ERR_SHAPE;
    if (p->io_dtype != SS_F32 && p->io_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if (p->flags & ~kGateFlags) return SS_ERR_UNSUPPORTED;
    const bool hi = p->flags & SS_GATE_HAS_I, hz = p->flags & SS_GATE_HAS_Z;
    if ((p->flags & SS_GATE_HAS_I_BIAS) && !hi) return SS_ERR_UNSUPPORTED;
    if ((long)p->batch * p->dim >= 0x7fffffffL || p->seqlen > 0x7fffffff - 4 * ss::GATE_PIECE) return SS_ERR_UNSUPPORTED;   // room for a team's last round
    if ((int64_t)p->batch * p->dim * ss::lanes_for(p->seqlen) > MOST_THREADS) return SS_ERR_UNSUPPORTED;
    const bool empty = p->seqlen == 0;
    if (!empty && (!p->x || !p->f || (hi && !p->i) || (hz && !p->z) || (!for_bwd && !p->out))) return SS_ERR_NULL;
    if (!p->rate || ((p->flags & SS_GATE_HAS_F_BIAS) && !p->f_bias) || ((p->flags & SS_GATE_HAS_I_BIAS) && !p->i_bias)) return SS_ERR_NULL;
    if (!empty && (p->flags & SS_GATE_HAS_RESET) && !p->reset) return SS_ERR_NULL;
    if ((p->flags & SS_GATE_HAS_H0) && !p->h0) return SS_ERR_NULL;
    if (!for_bwd && (p->flags & SS_GATE_WRITE_H_LAST) && !p->h_last) return SS_ERR_NULL;
    const int64_t dense = (int64_t)p->dim * p->seqlen;
    if (p->batch > 1 && (p->x_batch < dense || p->f_batch < dense || (hi && p->i_batch < dense) || (hz && p->z_batch < dense))) return SS_ERR_SHAPE;
    const size_t esz = p->io_dtype == SS_BF16 ? 2 : 4;
    if (!aligned_to(p->x, esz) || !aligned_to(p->f, esz) || (hi && !aligned_to(p->i, esz)) || (hz && !aligned_to(p->z, esz)) ||
        (!for_bwd && !aligned_to(p->out, esz)))
        return SS_ERR_ALIGN;
    if (!aligned_to(p->rate, 4) || !aligned_to(p->f_bias, 4) || !aligned_to(p->i_bias, 4) || !aligned_to(p->h0, 4) ||
        (!for_bwd && !aligned_to(p->h_last, 4)))
        return SS_ERR_ALIGN;
    return SS_OK;
}
GateArgs gate_args(const ss_gate_params* p, const GatePlan& g)
{
    GateArgs a{};
    a.B = p->batch; a.D = p->dim; a.L = p->seqlen; a.R = p->batch * p->dim;
    a.pieces = g.pieces; a.nseg = g.nseg; a.spp = g.spp; a.nmap = g.nmap; a.ppm = g.ppm;
    a.flags = p->flags;
    a.x = p->x; a.f = p->f; a.i = p->i; a.z = p->z;
    a.xb = p->x_batch; a.fb = p->f_batch; a.ib = p->i_batch; a.zb = p->z_batch;
    a.rate = p->rate; a.f_bias = p->f_bias; a.i_bias = p->i_bias; a.reset = p->reset; a.h0 = p->h0;
    return a;
}
void fill(float* to, const float* from, long n, hipStream_t st)
{
    hipLaunchKernelGGL(ss::gate_fill_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, to, from, (int)n);
}

}  // namespace

extern "C" {

size_t ss_gate_workspace_bytes(const ss_gate_params* p, int for_backward)
{
    if (!p || p->batch < 1 || p->dim < 1 || p->seqlen < 0) return 0;
    const long rows = (long)p->batch * p->dim;
    // the plan's io_dtype decides on the team's size alone, and where a row is split that is four either way
    return gate_space(rows, gate_plan(rows, p->seqlen, SS_F32), for_backward != 0).total;
}

int ss_gate_fwd(const ss_gate_params* p, void* stream)
{
    const int rc = check_gate(p, false);
    if (rc != SS_OK) return rc;
    const long rows = (long)p->batch * p->dim;
    const bool save = p->flags & SS_GATE_SAVE_FOR_BWD;
    GatePlan g = gate_plan(rows, p->seqlen, p->io_dtype);
    const GateSpace s = gate_space(rows, g, save);
    char* const ws = static_cast<char*>(p->workspace);
    if (ws && !aligned_to(ws, 256)) return SS_ERR_ALIGN;
    const bool have = ws && p->workspace_bytes >= s.total;
    if (save && s.total > 0 && !have) return SS_ERR_WORKSPACE;
    if (!have) {
        g.nseg = g.nmap = 1;
        g.spp = g.ppm = g.pieces;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    GateArgs a = gate_args(p, g);
    a.out = p->out;
    a.h_last = (p->flags & SS_GATE_WRITE_H_LAST) ? p->h_last : nullptr;
    if (p->seqlen == 0) {
        if (a.h_last) fill(a.h_last, (p->flags & SS_GATE_HAS_H0) ? p->h0 : nullptr, rows, st);
        return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
    }
    if (save) a.ckpt = reinterpret_cast<float*>(ws + s.ckpt);
    if (g.nseg > 1) {
        a.agg = reinterpret_cast<float2*>(ws + s.agg);
        a.carry = reinterpret_cast<float*>(ws + s.carry);
    }
    if (p->io_dtype == SS_BF16) ss::launch_all<ss::bf16_t>(a, g.team, false, st);
    else ss::launch_all<float>(a, g.team, false, st);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

int ss_gate_bwd(const ss_gate_bwd_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const ss_gate_params* q = &p->fwd;
    const int rc = check_gate(q, true);
    if (rc != SS_OK) return rc;
    const bool hi = q->flags & SS_GATE_HAS_I, hz = q->flags & SS_GATE_HAS_Z, fb = q->flags & SS_GATE_HAS_F_BIAS, ib = q->flags & SS_GATE_HAS_I_BIAS;
    const bool empty = q->seqlen == 0;
    if (!empty && (!p->dout || !p->dx || !p->df || (hi && !p->di) || (hz && !p->dz))) return SS_ERR_NULL;
    if (!p->drate || (fb && !p->df_bias) || (ib && !p->di_bias)) return SS_ERR_NULL;
    const int64_t dense = (int64_t)q->dim * q->seqlen;
    if (q->batch > 1 && (p->dx_batch < dense || p->df_batch < dense || (hi && p->di_batch < dense) || (hz && p->dz_batch < dense))) return SS_ERR_SHAPE;
    const size_t esz = q->io_dtype == SS_BF16 ? 2 : 4;
    if (!aligned_to(p->dout, esz) || !aligned_to(p->dx, esz) || !aligned_to(p->df, esz) || (hi && !aligned_to(p->di, esz)) ||
        (hz && !aligned_to(p->dz, esz)) || !aligned_to(p->dh_last, 4) || !aligned_to(p->drate, 4) || (fb && !aligned_to(p->df_bias, 4)) ||
        (ib && !aligned_to(p->di_bias, 4)) || !aligned_to(p->dh0, 4))
        return SS_ERR_ALIGN;
    const long rows = (long)q->batch * q->dim;
    const GatePlan g = gate_plan(rows, q->seqlen, q->io_dtype);
    const GateSpace s = gate_space(rows, g, true);
    char* const ws = static_cast<char*>(q->workspace);
    if (!empty && (!ws || q->workspace_bytes < s.total)) return SS_ERR_WORKSPACE;
    if (!aligned_to(ws, 256)) return SS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (empty) {
        fill(p->drate, nullptr, q->dim, st);
        if (fb) fill(p->df_bias, nullptr, q->dim, st);
        if (ib) fill(p->di_bias, nullptr, q->dim, st);
        if (p->dh0) fill(p->dh0, p->dh_last, rows, st);
        return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
    }
    GateArgs a = gate_args(q, g);
    a.ckpt = reinterpret_cast<float*>(ws + s.ckpt);
    if (g.nseg > 1) {
        a.agg = reinterpret_cast<float2*>(ws + s.agg);
        a.carry = reinterpret_cast<float*>(ws + s.carry);
    }
    a.dout = p->dout; a.dh_last = p->dh_last;
    a.dx = p->dx; a.df = p->df; a.di = p->di; a.dz = p->dz;
    a.dxb = p->dx_batch; a.dfb = p->df_batch; a.dib = p->di_batch; a.dzb = p->dz_batch;
    a.dh0 = p->dh0;
    // one segment of one batch entry: the rows' sums are the gradients
    const bool direct = g.nseg == 1 && q->batch == 1;
    const int64_t plane = (int64_t)g.nseg * rows;
    float* const part = reinterpret_cast<float*>(ws + s.part);
    a.part_rate = direct ? p->drate : part;
    a.part_f = fb ? (direct ? p->df_bias : part + plane) : nullptr;
    a.part_i = ib ? (direct ? p->di_bias : part + 2 * plane) : nullptr;
    if (q->io_dtype == SS_BF16) ss::launch_all<ss::bf16_t>(a, g.team, true, st);
    else ss::launch_all<float>(a, g.team, true, st);
    if (!direct)
        hipLaunchKernelGGL(ss::gate_sums_kernel, dim3((unsigned)std::min<int64_t>(((int64_t)q->dim + 15) / 16, MOST_THREADS / 256), ib ? 3u : (fb ? 2u : 1u)), dim3(256), 0, st, part, p->drate,
                           fb ? p->df_bias : nullptr, ib ? p->di_bias : nullptr, plane, q->dim, g.nseg * q->batch);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

int ss_gate_step(const ss_gate_step_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    if (p->batch < 1 || p->dim < 1) return SS_ERR_SHAPE;
    if (p->io_dtype != SS_F32 && p->io_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if (p->flags & ~kGateStepFlags) return SS_ERR_UNSUPPORTED;
    const bool hi = p->flags & SS_GATE_HAS_I, hz = p->flags & SS_GATE_HAS_Z;
    if ((p->flags & SS_GATE_HAS_I_BIAS) && !hi) return SS_ERR_UNSUPPORTED;
    const long n = (long)p->batch * p->dim;
    if (n >= 0x7fffffffL - 256) return SS_ERR_UNSUPPORTED;
    if (!p->h || !p->x_t || !p->f_t || (hi && !p->i_t) || (hz && !p->z_t) || !p->rate || !p->out_t) return SS_ERR_NULL;
    if (((p->flags & SS_GATE_HAS_F_BIAS) && !p->f_bias) || ((p->flags & SS_GATE_HAS_I_BIAS) && !p->i_bias)) return SS_ERR_NULL;
    if ((p->flags & SS_GATE_HAS_RESET) && !p->reset_t) return SS_ERR_NULL;
    if (p->batch > 1 && (p->x_batch < p->dim || p->f_batch < p->dim || (hi && p->i_batch < p->dim) || (hz && p->z_batch < p->dim))) return SS_ERR_SHAPE;
    const size_t esz = p->io_dtype == SS_BF16 ? 2 : 4;
    if (!aligned_to(p->h, 4) || !aligned_to(p->x_t, esz) || !aligned_to(p->f_t, esz) || (hi && !aligned_to(p->i_t, esz)) ||
        (hz && !aligned_to(p->z_t, esz)) || !aligned_to(p->rate, 4) || !aligned_to(p->f_bias, 4) || !aligned_to(p->i_bias, 4) || !aligned_to(p->out_t, esz))
        return SS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)((n + 255) / 256)), block(256);
    if (p->io_dtype == SS_BF16) hipLaunchKernelGGL(ss::gate_step_kernel<ss::bf16_t>, grid, block, 0, st, *p);
    else hipLaunchKernelGGL(ss::gate_step_kernel<float>, grid, block, 0, st, *p);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
