// Log probabilities of given tokens with the entropy and the most probable alternatives, and their gradient, for gfx950, with the C-ABI
// entry points (see include/ss_logprob.h).
//
// The logits are read once by each pass, and the gradient is written: both are bound by HBM.  Forward: every lane keeps the
// largest logit m that it has seen, S = sum exp(x - m) and U = sum exp(x - m) (x - m), which are brought to a new m by
// S <- c S, U <- c (U + S (m_old - m)) with c = exp(m_old - m); lanes, waves and workgroups are joined by the same rule.  Then
// lse = m + log S and the entropy log S - U / S.  Few rows are cut into pieces for several workgroups.
// Alternatives: a wave holds its best, in order, one a lane.  Of 64 groups of logits, one a lane, the top-th largest maximum is a bound below
// which nothing can be among the top, so of thousands of logits only about `top` are left; those are ranked among each other and the ones
// so far.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ss_logprob.h"
#include "ss_slices.h"

namespace ss {

struct LogprobArgs {
    int rows, vocab, top;
    int64_t row_stride;
    const void *logits, *targets;
    float *logp, *entropy, *max, *inv, *top_logp;
    int64_t* top_ids;
    int pieces, piece;        // workgroups of a row, columns of each
    int parts;                // what the waves of a row's workgroups leave
    float* part;              // (rows, parts): m, S, U and the best
    const float *dlogp, *dentropy;
    void* dlogits;
};

constexpr float FAR = -200.0f;   // exp of it is 0 in float32; a logarithm of a probability that is 0 is cut off here, so that 0 times it is 0

struct Stat {
    float m, s, u;
};
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
// what m is taken as where nothing but -infinity has been seen
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ void shift(Stat& a, float ref)
{
    const float d = fmaxf(a.m - ref, FAR), c = exp_of(d);
    a.u = (a.u + a.s * d) * c;
    a.s *= c;
}
__device__ __forceinline__ Stat join(Stat a, Stat b)
{
    const float m = fmaxf(a.m, b.m), ref = reference(m);
    shift(a, ref);
    shift(b, ref);
    return {m, a.s + b.s, a.u + b.u};
}
// The same over a wave, in all of its lanes: the largest first, then two sums of lanes that have been brought to it.  Lanes exchange by the vector
// unit's own means: within rows of 16, then the last lane of a row into the next row, and the last of the first half into the second.
template <int CONTROL, int ROWS>
__device__ __forceinline__ float from_lane(float v, float none)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(none), (int)__float_as_uint(v), CONTROL, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float over_wave(float v, float none, F op)
{
    v = op(v, from_lane<0x111, 0xf>(v, none));
    v = op(v, from_lane<0x112, 0xf>(v, none));
    v = op(v, from_lane<0x114, 0xf>(v, none));
    v = op(v, from_lane<0x118, 0xf>(v, none));
    v = op(v, from_lane<0x142, 0xa>(v, none));
    v = op(v, from_lane<0x143, 0xc>(v, none));
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), WAVE - 1));
}
__device__ __forceinline__ Stat join_wave(Stat a)
{
    const float m = over_wave(a.m, -INFINITY, [](float x, float y) { return fmaxf(x, y); });
    shift(a, reference(m));
    auto add = [](float x, float y) { return x + y; };
    return {m, over_wave(a.s, 0.0f, add), over_wave(a.u, 0.0f, add)};
}

// ---- the best of a wave ---------------------------------------------------------------------------
// A logit and its column as one number, whose order is theirs: the larger logit first, of equal ones the lower column.  0: none.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);   // zeros of both signs are equal
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }
__device__ __forceinline__ uint64_t rank_of(float v, int column) { return (uint64_t)order_of(v) << 32 | (uint32_t)~column; }
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// Lane l holds the l-th best.  All lanes call; `top` lanes are kept exact.  `room`: 64 places of the wave's own in LDS.
struct Best {
    uint64_t r = 0;
    __device__ __forceinline__ bool empty() const { return r == 0; }
    __device__ __forceinline__ float value() const { return logit_of((uint32_t)(r >> 32)); }
    __device__ __forceinline__ int column() const { return (int)~(uint32_t)r; }
    // The lanes' proposals, those of `ask`, take their places: every one is compared with all places and all others, none waits for another.
    __device__ __forceinline__ void merge(uint64_t proposal, uint64_t ask, uint64_t* room)
    {
        const int lane = threadIdx.x % WAVE;
        const bool mine = ask >> lane & 1;
        int place = lane, rank = 0, behind = 0;
#pragma unroll 1
        while (ask) {
            const int l = __ffsll((long long)ask) - 1;
            ask &= ask - 1;
            const uint64_t p = of_lane(proposal, l);
            place += p > r ? 1 : 0;
            rank += p > proposal ? 1 : 0;
            const int before = __popcll(__ballot(r > p));
            behind = lane == l ? before : behind;
        }
        rank += behind;
        room[lane] = 0;
        wave_lds_fence();
        if (r != 0 && place < WAVE) room[place] = r;
        if (mine && rank < WAVE) room[rank] = proposal;
        wave_lds_fence();
        r = room[lane];
        wave_lds_fence();
    }
    // What is no better has no place: the last of the top, or, as long as it is not full, what is below the top-th largest of the lanes' largest
    // (`most`, in its order, 0 where a lane has none), as that many are no less.  Its upper 16 bits are enough, found from the highest down.
    __device__ __forceinline__ uint64_t least(uint32_t most, int top) const
    {
        const uint64_t last = of_lane(r, top - 1);
        if (last) return last;
        uint32_t bound = 0;
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
            if (__popcll(__ballot(most >= (bound | bit))) >= top) bound |= bit;
        return bound ? ((uint64_t)bound << 32) - 1 : 0;
    }
    // of(j) of the lanes' open bits j take their places where they are above `than`: the first of every lane, then the second, ...
    template <typename F>
    __device__ __forceinline__ void absorb(uint32_t open, F of, uint64_t than, int top, uint64_t* room)
    {
#pragma unroll 1
        while (__ballot(open != 0)) {
            const uint64_t proposal = open ? of(__ffs((int)open) - 1) : 0, ask = __ballot(proposal > than);
            open &= open - 1;
            if (!ask) continue;
            merge(proposal, ask, room);
            than = max(than, of_lane(r, top - 1));
        }
    }
};

// ---- results of a row -----------------------------------------------------------------------------
template <typename I>
__device__ __forceinline__ int target_of(const LogprobArgs& a, int row)   // -1: none
{
    if (!a.targets) return -1;
    const I t = static_cast<const I*>(a.targets)[row];
    return t >= 0 && t < a.vocab ? (int)t : -1;
}
// The target's logit, requested before the row is done: 0 where there is none.
template <typename T, typename I>
__device__ __forceinline__ float target_logit(const LogprobArgs& a, int row, int target)
{
    return target < 0 ? 0.0f : io_to_f32<T>(static_cast<const T*>(a.logits)[row * a.row_stride + target]);
}
template <bool TOP>
__device__ __forceinline__ void results(const LogprobArgs& a, int row, Stat t, const Best& best, int target, float logit)
{
    const int lane = threadIdx.x % WAVE;
    const bool none = t.s == 0.0f;   // the largest logit alone makes S one
    const float ls = logf(t.s);
    auto logp = [&](float x) { return none ? -INFINITY : (x - t.m) - ls; };
    if (lane == 0) {
        if (a.logp) a.logp[row] = target < 0 ? 0.0f : logp(logit);
        a.entropy[row] = none ? 0.0f : ls - t.u / t.s;
        a.max[row] = none ? 0.0f : t.m;
        a.inv[row] = none ? 0.0f : 1.0f / t.s;
    }
    if constexpr (TOP) {
        if (lane < a.top) {
            a.top_logp[(int64_t)row * a.top + lane] = best.empty() ? __uint_as_float(0x7fc00000u) : logp(best.value());
            a.top_ids[(int64_t)row * a.top + lane] = best.empty() ? -1 : best.column();
        }
    }
}
// floats of a part of a row: m, S, U, then the `top` best, two each
__host__ __device__ __forceinline__ int part_floats(int top) { return 4 + 2 * top; }

// G lanes a row (a wave: rows side by side) or piece of one; V slices of eight a lane and step, the next step's requested ahead.  Bound by HBM: 8192 x
// 51200 bf16 (839 MB) 151 us, 5.6 TB/s (156 to 182 where a gradient has been written before); few rows by a launch and, with alternatives, by the
// lanes' choice: 64 x 51200 4.5 us, with eight 7.2.
template <typename T, typename I, int G, int V, bool TOP>
__global__ __launch_bounds__(256) void logprob_fwd_kernel(LogprobArgs a)
{
    constexpr int SIDE = 256 / G, WAVES = G / WAVE;
    const int gl = threadIdx.x % G;
    const unsigned group = blockIdx.x * SIDE + threadIdx.x / G;
    const int row = (int)(group / (unsigned)a.pieces), piece = (int)(group % (unsigned)a.pieces);
    if (row >= a.rows) return;   // a whole wave
    const T* x = static_cast<const T*>(a.logits) + row * a.row_stride;
    constexpr int STEP = V * G * 8;
    const int W = a.vocab, from = piece * a.piece, to = piece == a.pieces - 1 ? W : from + a.piece;   // the last's own end may lie behind 32 bits
    Stat t = {-INFINITY, 0.0f, 0.0f};
    Best best;
    __shared__ uint64_t room[TOP ? 4 : 1][WAVE];
    __shared__ float logits[TOP ? 4 : 1][V * 8][TOP ? WAVE : 1];   // a lane's, side by side with the others'
    // V slices of eight columns; those behind the piece are -infinity, and no candidates
    auto take = [&](const float (&f)[V][8], int base) {
        float m = t.m;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, f[v][j]);
        const float ref = reference(m);
        shift(t, ref);
        t.m = m;
        // A slice's values one after another, slices as a tree, and only then onto those of the steps before: all one by one, small terms that
        // together count are lost beside a large one (rows of 50021 with a few large logits: S off by 2.9e-7 in the mean, now by 0.75e-7).
        float se[V], su[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = f[v][j] - ref, e = exp_of(d);   // NaN stays NaN in e
                se[v] = j == 0 ? e : se[v] + e;
                su[v] = j == 0 ? e * fmaxf(d, FAR) : fmaf(e, fmaxf(d, FAR), su[v]);
            }
        }
        if constexpr (V == 4) {
            t.s += (se[0] + se[1]) + (se[2] + se[3]);
            t.u += (su[0] + su[1]) + (su[2] + su[3]);
        } else {
            t.s += se[0] + se[1];
            t.u += su[0] + su[1];
        }
        if constexpr (TOP) {
            const int lane = threadIdx.x % WAVE;
            float(*const all)[WAVE] = reinterpret_cast<float(*)[WAVE]>(logits[threadIdx.x / WAVE]);
            float most = -INFINITY;   // of what is no NaN; what is behind the piece is -infinity
            bool some = false;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    all[v * 8 + j][lane] = f[v][j];
                    some = some || f[v][j] == f[v][j];
                    most = fmaxf(most, f[v][j]);
                }
            const uint64_t than = best.least(some ? order_of(most) : 0u, a.top);
            const float low = than >> 32 >= 0x007fffffu ? logit_of((uint32_t)(than >> 32)) : -INFINITY;
            uint32_t open = 0;
#pragma unroll
            for (int j = 0; j < V * 8; ++j) open |= f[j / 8][j % 8] >= low ? 1u << j : 0u;
            best.absorb(open, [&](int j) {
                const int k = base + (j / 8 * G + gl) * 8 + j % 8;
                return k < to ? rank_of(all[j][lane], k) : 0;
            }, than, a.top, room[threadIdx.x / WAVE]);
        }
    };
    // whole steps, whose loads need no bounds and are requested a step ahead
    int base = from;
    if (base + STEP <= to) {
        typename io8<T>::raw raw[V];
        auto load = [&](int at) {
#pragma unroll
            for (int v = 0; v < V; ++v) raw[v] = io8<T>::load_elem(x + at + (v * G + gl) * 8, 0u);
        };
        load(base);
        for (; base + STEP <= to; base += STEP) {
            float f[V][8];
#pragma unroll
            for (int v = 0; v < V; ++v) io8<T>::unpack(raw[v], f[v]);
            load(min(base + STEP, to - STEP));
            take(f, base);
        }
    }
    if (base < to) {   // the rest; the columns behind the last whole eight one by one
        const int end = W / 8 * 8, slice = (end - base) / 8;
        const bool mine = slice % G == gl;
        float f[V][8], rest[8];
#pragma unroll
        for (int j = 0; j < 7; ++j) rest[j] = mine && end + j < W ? io_to_f32<T>(x[end + j]) : -INFINITY;
        rest[7] = -INFINITY;
        typename io8<T>::raw raw[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = base + (v * G + gl) * 8;
            if (at + 8 <= to) raw[v] = io8<T>::load_elem(x + at, 0u);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = base + (v * G + gl) * 8;
            io8<T>::unpack(raw[v], f[v]);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[v][j] = at + 8 <= to ? f[v][j] : (at == end ? rest[j] : -INFINITY);
        }
        take(f, base);
    }
    t = join_wave(t);
    const int lane = threadIdx.x % WAVE;
    auto leave = [&](int part) {
        float* p = a.part + ((int64_t)row * a.parts + part) * part_floats(a.top);
        if (lane == 0) {
            p[0] = t.m;
            p[1] = t.s;
            p[2] = t.u;
        }
        if constexpr (TOP) {
            if (lane < a.top) reinterpret_cast<uint64_t*>(p + 4)[lane] = best.r;
        }
    };
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x / WAVE;
        if (a.pieces > 1) return leave(piece * WAVES + wave);
        __shared__ Stat stats[WAVES];
        __shared__ uint64_t ranks[WAVES][TOP ? WAVE : 1];
        if (lane == 0) stats[wave] = t;
        if constexpr (TOP) ranks[wave][lane] = lane < a.top ? best.r : 0;
        __syncthreads();
        if (wave != 0) return;
        for (int w = 1; w < WAVES; ++w) t = join(t, stats[w]);
        if constexpr (TOP) {
            for (int w = 1; w < WAVES; ++w) {
                const uint64_t proposal = ranks[w][lane], ask = __ballot(proposal > of_lane(best.r, a.top - 1));
                if (ask) best.merge(proposal, ask, room[0]);
            }
        }
    }
    const int target = target_of<I>(a, row);
    results<TOP>(a, row, t, best, target, target_logit<T, I>(a, row, target));
}
// The parts of a row, a wave a row: two trips to memory, 3.5 us of 64 rows of seven pieces, with eight alternatives 5.
template <typename T, typename I, bool TOP>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a)
{
    const int row = blockIdx.x, lane = threadIdx.x;
    const int target = target_of<I>(a, row);
    const float* p = a.part + (int64_t)row * a.parts * part_floats(a.top);
    Stat t = {-INFINITY, 0.0f, 0.0f};
    for (int k = lane; k < a.parts; k += WAVE) {
        const float* q = p + (int64_t)k * part_floats(a.top);
        t = join(t, {q[0], q[1], q[2]});
    }
    const float logit = target_logit<T, I>(a, row, target);
    Best best;
    if constexpr (TOP) {
        constexpr int N = 8;
        __shared__ uint64_t room[WAVE], held[N][WAVE];
        const int all = a.parts * a.top;
#pragma unroll 1
        for (int c0 = 0; c0 < all; c0 += N * WAVE) {
            uint64_t v[N];
            uint32_t most = 0, open = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = c0 + j * WAVE + lane, part = min(c, all - 1) / a.top;
                const uint64_t r = reinterpret_cast<const uint64_t*>(p + (int64_t)part * part_floats(a.top) + 4)[min(c, all - 1) - part * a.top];
                v[j] = c < all ? r : 0;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                held[j][lane] = v[j];
                most = max(most, (uint32_t)(v[j] >> 32));
            }
            const uint64_t than = best.least(most, a.top);
#pragma unroll
            for (int j = 0; j < N; ++j) open |= v[j] > than ? 1u << j : 0u;
            best.absorb(open, [&](int j) { return held[j][lane]; }, than, a.top, room);
        }
    }
    results<TOP>(a, row, join_wave(t), best, target, logit);
}

// ---- backward -------------------------------------------------------------------------------------
// G lanes a row or piece of one, all of its slices requested at once.  PAST: the gradient goes past the caches.  Bound by HBM: 8192 x 51200 bf16 (1678 MB) 276 us,
// 6.1 TB/s (a part of the logits is in a cache from the forward pass); 777 x 50021 float32 (311 MB) 50, 6.2 TB/s.
template <typename T, typename I, int G, bool PAST>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobArgs a)
{
    constexpr int N = 16 / sizeof(T), V = 32 / N, SIDE = 256 / G;
    const int gl = threadIdx.x % G;
    const unsigned group = blockIdx.x * SIDE + threadIdx.x / G;
    // the last rows first: the forward pass, which has read them last, may have left them in a cache
    const int row = a.rows - 1 - (int)(group / (unsigned)a.pieces), from = (int)(group % (unsigned)a.pieces) * a.piece;
    if (row < 0) return;
    const int W = a.vocab, k = target_of<I>(a, row);
    const float inv = a.inv[row];
    const bool some = inv != 0.0f;   // also where it is NaN
    const float dl = a.dlogp && k >= 0 && some ? a.dlogp[row] : 0.0f, dh = a.dentropy && some ? a.dentropy[row] : 0.0f;
    T* out = static_cast<T*>(a.dlogits) + (int64_t)row * W;
    if (dl == 0.0f && dh == 0.0f) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = from + (v * G + gl) * N;
            if (at + N <= W) store_any(out + at, 0u, u32x4{0u, 0u, 0u, 0u});
            else {
                for (int j = 0; at + j < W; ++j) out[at + j] = (T)0;
            }
        }
        return;
    }
    const T* x = static_cast<const T*>(a.logits) + row * a.row_stride;
    const float m = a.max[row], ls = logf(inv);
    // dx = -p (dl + dh (log p + H)) = -p (c0 + dh d), d = x - m
    const float c0 = dh == 0.0f ? dl : fmaf(dh, ls + a.entropy[row], dl), c1 = -c0 * inv;
    auto gradient = [&](float (&f)[N], int at) {
        if (dh == 0.0f) {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = exp_of(f[j] - m) * c1;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = f[j] - m;
                f[j] = -(exp_of(d) * inv) * fmaf(dh, fmaxf(d, FAR), c0);
            }
        }
        if ((unsigned)(k - at) < (unsigned)N) {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] += at + j == k ? dl : 0.0f;
        }
    };
    u32x4 raw[V];
    float f[N];
    if (from + V * G * N <= W) {   // loads and stores need no bounds
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = load_any<u32x4>(x + from + (v * G + gl) * N, 0u);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = from + (v * G + gl) * N;
            words16<T>::unpack(raw[v], f);
            gradient(f, at);
            if constexpr (PAST) store_past(out + at, words16<T>::pack(f));
            else store_any(out + at, 0u, words16<T>::pack(f));
        }
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = from + (v * G + gl) * N;
        if (at + N <= W) raw[v] = load_any<u32x4>(x + at, 0u);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = from + (v * G + gl) * N;
        if (at >= W) break;
        const bool full = at + N <= W;
        if (full) words16<T>::unpack(raw[v], f);
        else {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = at + j < W ? io_to_f32<T>(x[at + j]) : 0.0f;
        }
        gradient(f, at);
        if (full) store_any(out + at, 0u, words16<T>::pack(f));
        else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (at + j < W) out[at + j] = f32_to_io<T>(f[j]);
        }
    }
}

// ---- sizes ----------------------------------------------------------------------------------------
constexpr int LOGPROB_STEP = 4 * 256 * 8;    // columns that a workgroup has in registers at once
constexpr int LOGPROB_WAVE = 4 * 64 * 8;     // and a wave: up to here a row is one wave's

struct LogprobPlan {
    int pieces, piece, parts;
    size_t bytes;
};
// Fewer than 256 rows are cut, for some 512 workgroups, into pieces of one step of a workgroup at least.  Of 51200 bf16 columns: 64 rows 4.5 us and
// 3.5 to join them, whole 7.2, with eight alternatives 7.4 and 4.8, whole 16.8; 256 rows whole 8.2, in two pieces 8.3 and 3.4; 512 whole 12.2, in
// four 12.8 and 4.2.  Smaller pieces: a wave's choice among its 2048 columns takes as long as their sums (64 rows with eight alternatives in pieces
// of 2048: 12.9 and 7.6).  The same with and without alternatives, so that the sums are the same to the bit.
LogprobPlan logprob_plan(int rows, int vocab, int top)
{
    LogprobPlan p = {1, vocab, 1, 0};
    if (vocab <= LOGPROB_WAVE || rows >= 256) return p;
    const int step = LOGPROB_STEP, units = (vocab + step - 1) / step, want = std::min({(512 + rows - 1) / rows, units, 1024});
    const int each = (units + want - 1) / want;
    p.piece = each * step;
    p.pieces = (units + each - 1) / each;
    p.parts = p.pieces * 4;
    if (p.pieces > 1) p.bytes = (size_t)rows * p.parts * part_floats(top) * sizeof(float);
    return p;
}

template <typename T, typename I, bool TOP>
void logprob_forward(const LogprobArgs& a, hipStream_t st)
{
    if (a.vocab <= LOGPROB_WAVE) {
        hipLaunchKernelGGL((logprob_fwd_kernel<T, I, 64, 2, TOP>), dim3((unsigned)(((int64_t)a.rows + 3) / 4)), dim3(256), 0, st, a);
        return;
    }
    const dim3 grid((unsigned)((int64_t)a.rows * a.pieces));
    hipLaunchKernelGGL((logprob_fwd_kernel<T, I, 256, 4, TOP>), grid, dim3(256), 0, st, a);
    if (a.pieces > 1) hipLaunchKernelGGL((logprob_join_kernel<T, I, TOP>), dim3((unsigned)a.rows), dim3(64), 0, st, a);
}
template <typename T, typename I, bool PAST>
void logprob_backward(LogprobArgs a, hipStream_t st)
{
    if (a.vocab <= LOGPROB_WAVE) {
        a.pieces = 1;
        a.piece = LOGPROB_WAVE;
        hipLaunchKernelGGL((logprob_bwd_kernel<T, I, 64, PAST>), dim3((unsigned)(((int64_t)a.rows + 3) / 4)), dim3(256), 0, st, a);
        return;
    }
    a.piece = LOGPROB_STEP;
    a.pieces = (a.vocab + LOGPROB_STEP - 1) / LOGPROB_STEP;
    hipLaunchKernelGGL((logprob_bwd_kernel<T, I, 256, PAST>), dim3((unsigned)((int64_t)a.rows * a.pieces)), dim3(256), 0, st, a);
}
template <typename F>
void with_types(const ss_logprob_params* p, F go)
{
    auto targets = [&](auto t) {
        if (p->flags & SS_LOGPROB_TARGETS_32) go(t, (int32_t)0);
        else go(t, (int64_t)0);
    };
    if (p->io_dtype == SS_F32) targets(float());
    else targets(bf16_t());
}

}  // namespace ss

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
constexpr int64_t LOGPROB_MOST = ((int64_t)1 << 24) - 1;   // workgroups of 256 threads: a launch has fewer than 2^32

int check_logprob(const ss_logprob_params* p)
{
    if (!p) return SS_ERR_NULL;
    if (p->rows < 0 || p->vocab < 1 || p->top < 0 || p->row_stride < p->vocab) return SS_ERR_SHAPE;
    if (p->io_dtype != SS_F32 && p->io_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if (p->flags & ~(uint32_t)SS_LOGPROB_TARGETS_32) return SS_ERR_UNSUPPORTED;
    if (p->top > p->vocab || p->top > SS_LOGPROB_MAX_TOP) return SS_ERR_UNSUPPORTED;
    if (p->vocab > 0x7fffffff - 65536) return SS_ERR_UNSUPPORTED;   // room for the last steps of the kernels' loops
    const int64_t pieces = p->vocab <= ss::LOGPROB_WAVE ? 1 : (p->vocab + ss::LOGPROB_STEP - 1) / ss::LOGPROB_STEP;
    if (p->rows * pieces > (p->vocab <= ss::LOGPROB_WAVE ? 4 * LOGPROB_MOST : LOGPROB_MOST)) return SS_ERR_UNSUPPORTED;
    if (p->rows > 0 && (!p->logits || !p->stats)) return SS_ERR_NULL;
    if (!aligned_to(p->logits, p->io_dtype == SS_BF16 ? 2 : 4) || !aligned_to(p->stats, 4)) return SS_ERR_ALIGN;
    if (!aligned_to(p->targets, p->flags & SS_LOGPROB_TARGETS_32 ? 4 : 8)) return SS_ERR_ALIGN;
    return SS_OK;
}
ss::LogprobArgs logprob_args(const ss_logprob_params* p)
{
    ss::LogprobArgs a{};
    a.rows = p->rows; a.vocab = p->vocab; a.top = p->top; a.row_stride = p->row_stride;
    a.logits = p->logits; a.targets = p->targets;
    a.entropy = p->entropy;
    a.max = p->stats;
    a.inv = p->stats + p->rows;
    return a;
}

}  // namespace

extern "C" {

size_t ss_logprob_workspace_bytes(const ss_logprob_params* p)
{
    if (!p || p->rows < 1 || p->vocab < 1 || p->top < 0 || p->top > SS_LOGPROB_MAX_TOP) return 0;
    return ss::logprob_plan(p->rows, p->vocab, p->top).bytes;
}

int ss_logprob_fwd(const ss_logprob_params* p, void* stream)
{
    const int rc = check_logprob(p);
    if (rc != SS_OK) return rc;
    if (p->rows == 0) return SS_OK;
    if (!p->entropy || (p->targets && !p->logp) || (p->top && (!p->top_logp || !p->top_ids))) return SS_ERR_NULL;
    if (!aligned_to(p->logp, 4) || !aligned_to(p->entropy, 4) || (p->top && (!aligned_to(p->top_logp, 4) || !aligned_to(p->top_ids, 8)))) return SS_ERR_ALIGN;
    const ss::LogprobPlan plan = ss::logprob_plan(p->rows, p->vocab, p->top);
    if (plan.bytes) {
        if (!p->workspace || p->workspace_bytes < plan.bytes) return SS_ERR_WORKSPACE;
        if (!aligned_to(p->workspace, 256)) return SS_ERR_ALIGN;
    }
    ss::LogprobArgs a = logprob_args(p);
    a.logp = p->logp;
    a.top_logp = p->top_logp; a.top_ids = p->top_ids;
    a.pieces = plan.pieces; a.piece = plan.piece; a.parts = plan.parts;
    a.part = static_cast<float*>(p->workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    ss::with_types(p, [&](auto t, auto i) {
        if (p->top) ss::logprob_forward<decltype(t), decltype(i), true>(a, st);
        else ss::logprob_forward<decltype(t), decltype(i), false>(a, st);
    });
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

int ss_logprob_bwd(const ss_logprob_bwd_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const ss_logprob_params* f = &p->fwd;
    const int rc = check_logprob(f);
    if (rc != SS_OK) return rc;
    if (f->rows == 0) return SS_OK;
    if (!p->dlogits || (p->dentropy && !f->entropy)) return SS_ERR_NULL;
    if (!aligned_to(p->dlogits, f->io_dtype == SS_BF16 ? 2 : 4) || !aligned_to(p->dlogp, 4) || !aligned_to(p->dentropy, 4) || !aligned_to(f->entropy, 4))
        return SS_ERR_ALIGN;
    ss::LogprobArgs a = logprob_args(f);
    a.dlogp = p->dlogp; a.dentropy = p->dentropy;
    a.dlogits = p->dlogits;
    hipStream_t st = static_cast<hipStream_t>(stream);
    ss::with_types(f, [&](auto t, auto i) {
        if ((int64_t)f->rows * f->vocab * (int64_t)sizeof(t) > ss::STREAM_BYTES) ss::logprob_backward<decltype(t), decltype(i), true>(a, st);
        else ss::logprob_backward<decltype(t), decltype(i), false>(a, st);
    });
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
