// Layer norm with the residual sum before it, forward and backward, for gfx950, with the C-ABI entry
// points (see include/ss_norm.h).
//
// Both passes move a few values per element and compute about ten operations on each, so they are bound by HBM and
// every tensor is touched once: a row is held in the registers of the G lanes that share it, the mean is taken, then the variance
// about that mean (two sweeps over registers, exact to float32 where a sum of squares would cancel), then the result is
// formed.  A group of lanes walks rows with the weights of its columns in registers.  The backward pass keeps its columns' sums
// for dweight and dbias in registers as well; a workgroup's go to the workspace and a second kernel adds them up in a fixed order.
#include <hip/hip_runtime.h>
#include <cmath>
#include <type_traits>

#include "ss_norm.h"
#include "ss_slices.h"

namespace ss {

struct NormArgs {
    int rows, width;
    float eps;
    const void *x, *residual;
    const float *weight, *bias;
    void *out, *summed;
    float *mean, *rstd;
    const void *s, *dout, *dsummed;
    void *dx, *dresidual;
    float *dweight, *dbias;
    float* part;   // (parts, 2, width)
};

// ---- sums over the G lanes of a row -----------------------------------------------------------
// 16 or 64 lanes: within the wave.  More: the waves' sums through LDS, whose two halves are used in turn, so one barrier a sum.
template <int G, int N>
struct RowSum {
    static constexpr int WAVES = G > WAVE ? G / WAVE : 1;
    float (*lds)[N][WAVES];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int s = 1; s < (G < WAVE ? G : WAVE); s *= 2) v[k] += __shfl_xor(v[k], s);
        if constexpr (G > WAVE) {
            if (threadIdx.x % WAVE == 0)
#pragma unroll
                for (int k = 0; k < N; ++k) lds[turn][k][threadIdx.x / WAVE] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float t = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) t += lds[turn][k][w];
                v[k] = t;
            }
            turn ^= 1;
        }
    }
};

// Threads of a workgroup and the rows it works on side by side.
template <int G> constexpr int norm_threads(bool bwd) { return G > WAVE ? G : (bwd ? 512 : 256); }
// The next row is requested before this one is worked on, but with 1024 lanes, which have 128 registers each (the backward kernels spill
// of them: 3 to 5 in float32, 14 to 22 in bf16 and with a float32 residual).
template <int G> constexpr bool norm_ahead() { return G < 1024; }

__device__ __forceinline__ void load_columns(const float* p, int at, int width, float none, float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = none;
    if (!p) return;
    if (at + 8 <= width) {
        io8<float>::unpack(io8<float>::load_elem(p + at, 0u), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + j < width) v[j] = p[at + j];
    }
}

// Lane l of the G of a row has slices l, l + G, ... (V of them).  At the rate of a large copy (5.15 TB/s): 16384 x 2048 bf16 with a
// residual of float32 (403 MB) 79 us, of bf16 (268 MB) 47; 2048 x 16384 (134 MB) 27.  One row of 2048 is a launch, 2.6 us.
template <typename T, typename S, int G, int V, bool RES>
__global__ __launch_bounds__(norm_threads<G>(false)) void norm_fwd_kernel(NormArgs a)
{
    constexpr int THREADS = norm_threads<G>(false), SIDE = THREADS / G;
    __shared__ float lds[2][1][RowSum<G, 1>::WAVES];
    RowSum<G, 1> sum{lds};
    const int gl = threadIdx.x % G, W = a.width;
    float w[V][8], b[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = (v * G + gl) * 8;
        load_columns(a.weight, at, W, 1.0f, w[v]);
        load_columns(a.bias, at, W, 0.0f, b[v]);
    }
    const float inv_w = 1.0f / (float)W;
    const int step = gridDim.x * SIDE;
    typename io8<T>::raw rx[V];
    typename io8<S>::raw rr[V];
    auto load = [&](int row) {
        row = min(row, a.rows - 1);
        const int limit = slice_limit(W, slice_whole(W, row == a.rows - 1));
        const T* x = static_cast<const T*>(a.x) + (int64_t)row * W;
        const S* r = static_cast<const S*>(a.residual) + (int64_t)row * W;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = (v * G + gl) * 8;
            rx[v] = slice_request<T, G == 16>(x, at, W, limit);
            if constexpr (RES) rr[v] = slice_request<S, G == 16>(r, at, W, limit);
        }
    };
    // G > 64: all lanes of the workgroup share the row, so they leave the loop together (the sums hold barriers); else rows
    // past the end are worked on with the last one's values and not stored
    const int first = blockIdx.x * SIDE + threadIdx.x / G;
    if constexpr (norm_ahead<G>()) load(first);
    for (int row = first; row - (int)(threadIdx.x / G) < a.rows; row += step) {
        if constexpr (!norm_ahead<G>()) load(row);
        float s[V][8];
        const bool valid = row < a.rows, whole = slice_whole(W, row >= a.rows - 1);
        if (!whole) {
            const int limit = slice_limit(W, false);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                slice_settle<T>(rx[v], (v * G + gl) * 8, W, limit, false);
                if constexpr (RES) slice_settle<S>(rr[v], (v * G + gl) * 8, W, limit, false);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            io8<T>::unpack(rx[v], s[v]);
            if constexpr (RES) {
                float r[8];
                io8<S>::unpack(rr[v], r);
                // what is held is what is normalised: rounded to the residual's type
#pragma unroll
                for (int j = 0; j < 8; ++j) s[v][j] += r[j];
                if constexpr (sizeof(S) == 2) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[v][j] = bf16_to_f32(f32_to_io<bf16_t>(s[v][j]));
                }
            }
        }
        if constexpr (norm_ahead<G>())
            if (row + step - (int)(threadIdx.x / G) < a.rows) load(row + step);
        float t[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = W - (v * G + gl) * 8;
            if (n < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[v][j] = j < n ? s[v][j] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) t[0] += s[v][j];
        }
        sum(t);
        const float mean = t[0] * inv_w;
        t[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int n = W - (v * G + gl) * 8;
            if (n >= 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[0] = fmaf(s[v][j] - mean, s[v][j] - mean, t[0]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[0] += j < n ? (s[v][j] - mean) * (s[v][j] - mean) : 0.0f;
            }
        }
        sum(t);
        const float rstd = 1.0f / sqrtf(t[0] * inv_w + a.eps);
        if (valid) {
            T* out = static_cast<T*>(a.out) + (int64_t)row * W;
            S* held = static_cast<S*>(a.summed) + (int64_t)row * W;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int at = (v * G + gl) * 8, n = W - at;
                if constexpr (RES) slice_store<S>(held, at, n, s[v]);
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = fmaf((s[v][j] - mean) * rstd, w[v][j], b[v][j]);
                slice_store<T>(out, at, n, o);
            }
            if (a.mean && gl == 0) {
                a.mean[row] = mean;
                a.rstd[row] = rstd;
            }
        }
    }
}

// With g = dout w and xh the normalised row: ds = rstd (g - mean g - xh mean(g xh)) + dsummed, two sums a row in one exchange; dweight
// and dbias are sums over rows of dout xh and dout.  Bound by HBM: 16384 x 2048 bf16 with residual (268 MB) 47 us, 5.7 TB/s; 5199 x 1021
// float32 (64 MB) 16 us, 4.0 TB/s (a wave has three rows, the first and last of which overlap with nothing); 2048 x 16384 (201 MB) 44.
template <typename T, typename S, int G, int V, bool RES>
__global__ __launch_bounds__(norm_threads<G>(true)) void norm_bwd_kernel(NormArgs a)
{
    constexpr int THREADS = norm_threads<G>(true), SIDE = THREADS / G;
    __shared__ float lds[2][2][RowSum<G, 2>::WAVES];
    RowSum<G, 2> sum{lds};
    const int gl = threadIdx.x % G, W = a.width;
    float w[V][8], dw[V][8], db[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        load_columns(a.weight, (v * G + gl) * 8, W, 1.0f, w[v]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[v][j] = db[v][j] = 0.0f;
    }
    const float inv_w = 1.0f / (float)W;
    const int step = gridDim.x * SIDE;
    const bool more = RES && a.dsummed;
    typename io8<S>::raw rs[V], rm[V];
    typename io8<T>::raw rd[V];
    float mean_next, rstd_next;
    auto load = [&](int row) {
        row = min(row, a.rows - 1);
        const int limit = slice_limit(W, slice_whole(W, row == a.rows - 1));
        const int64_t off = (int64_t)row * W;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = (v * G + gl) * 8;
            rs[v] = slice_request<S, G == 16>(static_cast<const S*>(a.s) + off, at, W, limit);
            rd[v] = slice_request<T, G == 16>(static_cast<const T*>(a.dout) + off, at, W, limit);
            if constexpr (RES && norm_ahead<G>())
                if (more) rm[v] = slice_request<S, G == 16>(static_cast<const S*>(a.dsummed) + off, at, W, limit);
        }
        mean_next = a.mean[row];
        rstd_next = a.rstd[row];
    };
    const int first = blockIdx.x * SIDE + threadIdx.x / G;
    if constexpr (norm_ahead<G>()) load(first);
    for (int row = first; row - (int)(threadIdx.x / G) < a.rows; row += step) {
        if constexpr (!norm_ahead<G>()) load(row);
        const bool valid = row < a.rows;
        const float mean = mean_next, rstd = rstd_next;
        float x[V][8], g[V][8], m[V][8];
        float t[2] = {0.0f, 0.0f};
        if (!slice_whole(W, row >= a.rows - 1)) {
            const int limit = slice_limit(W, false);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                slice_settle<S>(rs[v], (v * G + gl) * 8, W, limit, false);
                slice_settle<T>(rd[v], (v * G + gl) * 8, W, limit, false);
                if constexpr (RES && norm_ahead<G>())
                    if (more) slice_settle<S>(rm[v], (v * G + gl) * 8, W, limit, false);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            io8<S>::unpack(rs[v], x[v]);
            io8<T>::unpack(rd[v], g[v]);
            if constexpr (RES && norm_ahead<G>()) {   // the next row's come into the same registers
                if (more) io8<S>::unpack(rm[v], m[v]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) m[v][j] = 0.0f;
                }
            }
            const int n = valid ? W - (v * G + gl) * 8 : 0;
            if (n < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[v][j] = j < n ? x[v][j] : mean;
                    g[v][j] = j < n ? g[v][j] : 0.0f;
                }
            }
        }
        if constexpr (norm_ahead<G>())
            if (row + step - (int)(threadIdx.x / G) < a.rows) load(row + step);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[v][j] = (x[v][j] - mean) * rstd;
                dw[v][j] = fmaf(g[v][j], x[v][j], dw[v][j]);
                db[v][j] += g[v][j];
                g[v][j] *= w[v][j];
                t[0] += g[v][j];
                t[1] = fmaf(g[v][j], x[v][j], t[1]);
            }
        sum(t);
        const float c1 = t[0] * inv_w, c2 = t[1] * inv_w;
        if (valid) {
            const int64_t off = (int64_t)row * W;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int at = (v * G + gl) * 8, n = W - at;
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    o[j] = rstd * (g[v][j] - c1 - x[v][j] * c2);
                    if constexpr (RES && norm_ahead<G>()) o[j] += m[v][j];
                }
                if constexpr (RES && !norm_ahead<G>()) {
                    if (more) {
                        float mv[8];
                        const bool whole = slice_whole(W, row == a.rows - 1);
                        typename io8<S>::raw r = slice_request<S, false>(static_cast<const S*>(a.dsummed) + off, at, W, slice_limit(W, whole));
                        slice_settle<S>(r, at, W, slice_limit(W, whole), whole);
                        io8<S>::unpack(r, mv);
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] += mv[j];
                    }
                }
                slice_store<T>(static_cast<T*>(a.dx) + off, at, n, o);
                if constexpr (RES && sizeof(S) != sizeof(T)) slice_store<S>(static_cast<S*>(a.dresidual) + off, at, n, o);
            }
        }
    }
    // the workgroup's sums: groups of a wave by shuffles, then wave after wave through LDS
    if constexpr (G < WAVE) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int s = G; s < WAVE; s *= 2) {
                    dw[v][j] += __shfl_xor(dw[v][j], s);
                    db[v][j] += __shfl_xor(db[v][j], s);
                }
    }
    float* const part = a.part + (int64_t)blockIdx.x * 2 * W;
    if constexpr (G > WAVE) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = (v * G + gl) * 8, n = W - at;
            slice_store<float>(part, at, n, dw[v]);
            slice_store<float>(part + W, at, n, db[v]);
        }
    } else {
        constexpr int COLS = G * V * 8, WAVES = THREADS / WAVE;
        __shared__ float all[2][COLS];
        for (int k = 0; k < WAVES; ++k) {
            if (threadIdx.x / WAVE == (unsigned)k && threadIdx.x % WAVE < G) {
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int c = (v * G + gl) * 8 + j;
                        all[0][c] = k == 0 ? dw[v][j] : all[0][c] + dw[v][j];
                        all[1][c] = k == 0 ? db[v][j] : all[1][c] + db[v][j];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < W; c += THREADS) {
            part[c] = all[0][c];
            part[W + c] = all[1][c];
        }
    }
}

// dweight and dbias from the parts: 32 columns of one of the two per workgroup and round, 32 threads a column.  512 parts of 2048 columns 4.0 us.
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* part, float* dweight, float* dbias, int W, int parts)
{
    float* const to = blockIdx.y == 0 ? dweight : dbias;
    if (!to) return;
    __shared__ float s[32][33];
    const int k0 = threadIdx.x / 32;
    for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < W; c0 += (int64_t)gridDim.x * 32) {
        const int64_t c = c0 + threadIdx.x % 32;
        float v = 0.0f;
        if (c < W) {
#pragma unroll 8
            for (int k = k0; k < parts; k += 32) v += part[((int64_t)k * 2 + blockIdx.y) * W + c];
        }
        s[threadIdx.x % 32][k0] = v;
        __syncthreads();
        // a column's 32 sums in the lanes of half a wave
        float t = s[threadIdx.x / 32][threadIdx.x % 32];
#pragma unroll
        for (int k = 1; k < 32; k *= 2) t += __shfl_xor(t, k);
        const int64_t col = c0 + threadIdx.x / 32;
        if (threadIdx.x % 32 == 0 && col < W) to[col] = t;
        __syncthreads();
    }
}

// ---- rows that do not fit the registers of a workgroup ------------------------------------------
// A workgroup a row at a time, which is read once for each sweep, after the first from the caches.  An element a thread and access, which
// is what bounds them: 2048 x 20000 bf16 (164 MB), not in a cache, 101 us forward and 143 a backward call (float32 127 and 211); in a cache 80 and
// 115.  Kept simple, as rows this wide are few.
template <typename T, typename S, bool RES>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(NormArgs a)
{
    __shared__ float lds[2][1][16];
    RowSum<1024, 1> sum{lds};
    const int W = a.width;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t off = row * W;
        const T* x = static_cast<const T*>(a.x) + off;
        const S* r = static_cast<const S*>(a.residual) + off;
        S* held = static_cast<S*>(a.summed) + off;
        T* out = static_cast<T*>(a.out) + off;
        auto value = [&](int c) {
            if constexpr (RES) return io_to_f32<S>(held[c]);   // as this thread wrote it
            else return io_to_f32<T>(x[c]);
        };
        float t[1] = {0.0f};
        for (int c = threadIdx.x; c < W; c += 1024) {
            if constexpr (RES) held[c] = f32_to_io<S>(io_to_f32<T>(x[c]) + io_to_f32<S>(r[c]));
            t[0] += value(c);
        }
        sum(t);
        const float mean = t[0] / (float)W;
        t[0] = 0.0f;
        for (int c = threadIdx.x; c < W; c += 1024) {
            const float v = value(c) - mean;
            t[0] = fmaf(v, v, t[0]);
        }
        sum(t);
        const float rstd = 1.0f / sqrtf(t[0] / (float)W + a.eps);
        for (int c = threadIdx.x; c < W; c += 1024)
            out[c] = f32_to_io<T>(fmaf((value(c) - mean) * rstd, a.weight ? a.weight[c] : 1.0f, a.bias ? a.bias[c] : 0.0f));
        if (a.mean && threadIdx.x == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}
template <typename T, typename S, bool RES>
__global__ __launch_bounds__(1024) void norm_bwd_wide_kernel(NormArgs a)
{
    __shared__ float lds[2][2][16];
    RowSum<1024, 2> sum{lds};
    const int W = a.width;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t off = row * W;
        const S *s = static_cast<const S*>(a.s) + off, *more = static_cast<const S*>(a.dsummed) + off;
        const T* dout = static_cast<const T*>(a.dout) + off;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float t[2] = {0.0f, 0.0f};
        for (int c = threadIdx.x; c < W; c += 1024) {
            const float g = io_to_f32<T>(dout[c]) * (a.weight ? a.weight[c] : 1.0f);
            t[0] += g;
            t[1] = fmaf(g, (io_to_f32<S>(s[c]) - mean) * rstd, t[1]);
        }
        sum(t);
        const float c1 = t[0] / (float)W, c2 = t[1] / (float)W;
        for (int c = threadIdx.x; c < W; c += 1024) {
            const float g = io_to_f32<T>(dout[c]) * (a.weight ? a.weight[c] : 1.0f);
            float o = rstd * (g - c1 - (io_to_f32<S>(s[c]) - mean) * rstd * c2);
            if (RES && a.dsummed) o += io_to_f32<S>(more[c]);
            static_cast<T*>(a.dx)[off + c] = f32_to_io<T>(o);
            if constexpr (RES && sizeof(S) != sizeof(T)) static_cast<S*>(a.dresidual)[off + c] = o;
        }
    }
}
// columns' sums over blockIdx.y's share of the rows
template <typename T, typename S>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.0f, db = 0.0f;
    for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const int64_t e = (int64_t)row * a.width + c;
        const float g = io_to_f32<T>(static_cast<const T*>(a.dout)[e]);
        dw = fmaf(g, (io_to_f32<S>(static_cast<const S*>(a.s)[e]) - a.mean[row]) * a.rstd[row], dw);
        db += g;
    }
    float* const part = a.part + (int64_t)blockIdx.y * 2 * a.width;
    part[c] = dw;
    part[a.width + c] = db;
}

// ---- forms ----------------------------------------------------------------------------------------
constexpr int NORM_WIDEST = 16384;   // widest row that is held in registers
constexpr int NORM_MOST_WORKGROUPS = (1 << 22) - 1;   // of 1024 threads: a launch has fewer than 2^32

struct NormForm {
    int lanes, slices;   // lanes of a row (0: the kernels for wider rows) and slices of a lane
};
// One wave a row where there are rows enough to fill the chip with and its registers hold it (forward 2048 columns, backward
// 1024, which has three more values a column; 16 lanes up to 128 columns); more lanes a row for wider ones, and where rows are few.
NormForm norm_form(int rows, int width, bool bwd)
{
    auto slices = [&](int lanes) { const int n = (width + 8 * lanes - 1) / (8 * lanes); return n <= 1 ? 1 : (n <= 2 ? 2 : 4); };
    if (width > NORM_WIDEST) return {0, 0};
    if (width <= 16 * 8) return {16, 1};
    if (width <= 64 * 8) return {64, 1};
    if (width <= (bwd ? 64 * 16 : 64 * 32) && rows >= 1024) return {64, slices(64)};
    if (width <= (bwd ? 256 * 16 : 256 * 32)) return {256, slices(256)};
    if (bwd && width <= 512 * 16) return {512, 2};
    return {1024, 2};
}
template <bool BWD, typename F>
void with_form(NormForm f, F go)
{
    auto lanes = [&](auto g) {
        constexpr int G = decltype(g)::value;
        if constexpr (G <= 16) go(g, std::integral_constant<int, 1>{});
        else if constexpr (G > 256) go(g, std::integral_constant<int, 2>{});
        else {
            if (f.slices == 1) go(g, std::integral_constant<int, 1>{});
            else if (f.slices == 2) go(g, std::integral_constant<int, 2>{});
            else if constexpr (!BWD) go(g, std::integral_constant<int, 4>{});
        }
    };
    if (f.lanes == 16) lanes(std::integral_constant<int, 16>{});
    else if (f.lanes == 64) lanes(std::integral_constant<int, 64>{});
    else if (f.lanes == 256) lanes(std::integral_constant<int, 256>{});
    else if (f.lanes == 1024) lanes(std::integral_constant<int, 1024>{});
    else if constexpr (BWD) lanes(std::integral_constant<int, 512>{});
}
// Workgroups of a backward call, each with a row of partial sums: one or two for a unit, as each costs 8 bytes a column twice, and
// counts between leave units idle at the end.  us of a call with 128 / 256 / 384 / 512 / 768 (rows x columns, no residual): bf16 16384 x 1024 27.4 22.9
// 27.8 27.3 31.4, 2048 x 16384 67.5 55.3 67.4 71.2 86.0, 500 x 8192 16.6 19.6 21.0 24.2 23.9, 2048 x 2048 20.8 15.1 15.5 15.0 16.9; workgroups of 256 lanes are too
// few to keep memory busy then: 16384 x 2048 113 62.6 52.0 43.2 39.4, 8192 x 4096 81.1 48.5 45.4 44.2 45.1 (float32 134 80.3 84.3 78.5
// 81.8 and 111 78.8 87.3 82.5 85.3).  512 for both types and all rows from 4096 on:
// the least over these four together, though 768 (251.6 us against 248.4) is ahead in the first.
int norm_parts(int rows, int width)
{
    const NormForm f = norm_form(rows, width, true);
    if (f.lanes == 0) return rows < 64 ? rows : 64;
    const int side = f.lanes > WAVE ? 1 : 512 / f.lanes;
    const int n = (rows + side - 1) / side;
    const int most = f.lanes == 256 && rows >= 4096 ? 512 : (width > 4096 && rows < 1024 ? 128 : 256);
    return n < most ? n : most;
}

template <typename T, typename S, bool RES>
void norm_launch(const NormArgs& a, bool bwd, hipStream_t st)
{
    const NormForm f = norm_form(a.rows, a.width, bwd);
    if (f.lanes == 0) {
        const dim3 grid((unsigned)(a.rows < NORM_MOST_WORKGROUPS ? a.rows : NORM_MOST_WORKGROUPS));
        if (!bwd) {
            hipLaunchKernelGGL((norm_fwd_wide_kernel<T, S, RES>), grid, dim3(1024), 0, st, a);
        } else {
            hipLaunchKernelGGL((norm_bwd_wide_kernel<T, S, RES>), grid, dim3(1024), 0, st, a);
            if (a.part)
                hipLaunchKernelGGL((norm_columns_kernel<T, S>), dim3((unsigned)((a.width + 255) / 256), (unsigned)norm_parts(a.rows, a.width)),
                                   dim3(256), 0, st, a);
        }
        return;
    }
    if (bwd) {
        with_form<true>(f, [&](auto g, auto v) {
            constexpr int G = decltype(g)::value, V = decltype(v)::value;
            hipLaunchKernelGGL((norm_bwd_kernel<T, S, G, V, RES>), dim3((unsigned)norm_parts(a.rows, a.width)), dim3(norm_threads<G>(true)), 0, st, a);
        });
    } else {
        with_form<false>(f, [&](auto g, auto v) {
            constexpr int G = decltype(g)::value, V = decltype(v)::value;
            // workgroups of 1024 lanes, which request no row ahead, have two rounds of the units' at most (2048 x 16384 float32 53 us, four 62)
            const int side = norm_threads<G>(false) / G, n = (a.rows + side - 1) / side, most = G < 1024 ? 1024 : 512;
            hipLaunchKernelGGL((norm_fwd_kernel<T, S, G, V, RES>), dim3((unsigned)(n < most ? n : most)), dim3(norm_threads<G>(false)), 0, st, a);
        });
    }
}
void norm_dispatch(const NormArgs& a, int io, uint32_t flags, bool bwd, hipStream_t st)
{
    const bool res = flags & SS_NORM_HAS_RESIDUAL;
    if (io == SS_F32) {
        if (res) norm_launch<float, float, true>(a, bwd, st);
        else norm_launch<float, float, false>(a, bwd, st);
    } else if (!res) norm_launch<bf16_t, bf16_t, false>(a, bwd, st);
    else if (flags & SS_NORM_RESIDUAL_F32) norm_launch<bf16_t, float, true>(a, bwd, st);
    else norm_launch<bf16_t, bf16_t, true>(a, bwd, st);
}

}  // namespace ss

namespace {

constexpr uint32_t kNormFlags = SS_NORM_HAS_WEIGHT | SS_NORM_HAS_BIAS | SS_NORM_HAS_RESIDUAL | SS_NORM_RESIDUAL_F32 | SS_NORM_SAVE_STATS;
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct NormSizes {
    size_t io, held;   // bytes of an element of x, and of the sum
};
int check_norm(const ss_norm_params* p, NormSizes& e, bool for_bwd)
{
    if (!p) return SS_ERR_NULL;
    if (p->rows < 0 || p->width < 1) return SS_ERR_SHAPE;
    if (p->io_dtype != SS_F32 && p->io_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if (p->flags & ~kNormFlags) return SS_ERR_UNSUPPORTED;
    if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return SS_ERR_UNSUPPORTED;
    if (p->width > 0x7fffffff - 65536 || p->rows > 0x7fffffff - 65536) return SS_ERR_UNSUPPORTED;   // room for the last steps of the kernels' loops
    e.io = p->io_dtype == SS_BF16 ? 2 : 4;
    e.held = (p->flags & SS_NORM_HAS_RESIDUAL) && (p->flags & SS_NORM_RESIDUAL_F32) ? 4 : e.io;
    const bool hw = p->flags & SS_NORM_HAS_WEIGHT, hb = (p->flags & SS_NORM_HAS_BIAS) && !for_bwd;   // the bias's values are the forward pass's alone
    if ((hw && !p->weight) || (hb && !p->bias)) return SS_ERR_NULL;
    if ((hw && !aligned_to(p->weight, 4)) || (hb && !aligned_to(p->bias, 4))) return SS_ERR_ALIGN;
    return SS_OK;
}
ss::NormArgs norm_args(const ss_norm_params* p)
{
    ss::NormArgs a{};
    a.rows = p->rows; a.width = p->width; a.eps = p->eps;
    a.weight = (p->flags & SS_NORM_HAS_WEIGHT) ? p->weight : nullptr;
    a.bias = (p->flags & SS_NORM_HAS_BIAS) ? p->bias : nullptr;
    return a;
}

}  // namespace

extern "C" {

int ss_norm_fwd(const ss_norm_params* p, void* stream)
{
    NormSizes e;
    const int rc = check_norm(p, e, false);
    if (rc != SS_OK) return rc;
    const bool res = p->flags & SS_NORM_HAS_RESIDUAL, save = p->flags & SS_NORM_SAVE_STATS;
    if (p->rows == 0) return SS_OK;
    if (!p->x || !p->out || (res && (!p->residual || !p->summed)) || (save && !p->stats)) return SS_ERR_NULL;
    if (!aligned_to(p->x, e.io) || !aligned_to(p->out, e.io) || (res && (!aligned_to(p->residual, e.held) || !aligned_to(p->summed, e.held))) ||
        (save && !aligned_to(p->stats, 4)))
        return SS_ERR_ALIGN;
    ss::NormArgs a = norm_args(p);
    a.x = p->x; a.residual = p->residual; a.out = p->out; a.summed = p->summed;
    if (save) {
        a.mean = p->stats;
        a.rstd = p->stats + p->rows;
    }
    ss::norm_dispatch(a, p->io_dtype, p->flags, false, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

size_t ss_norm_workspace_bytes(const ss_norm_params* p)
{
    if (!p || p->rows < 1 || p->width < 1) return 0;
    return (size_t)ss::norm_parts(p->rows, p->width) * 2 * p->width * sizeof(float);
}

int ss_norm_bwd(const ss_norm_bwd_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const ss_norm_params* q = &p->fwd;
    NormSizes e;
    const int rc = check_norm(q, e, true);
    if (rc != SS_OK) return rc;
    const bool res = q->flags & SS_NORM_HAS_RESIDUAL, hw = q->flags & SS_NORM_HAS_WEIGHT, hb = q->flags & SS_NORM_HAS_BIAS;
    const void* s = res ? q->summed : q->x;
    const bool two = res && e.held != e.io;
    if ((hw && !p->dweight) || (hb && !p->dbias)) return SS_ERR_NULL;
    if ((hw && !aligned_to(p->dweight, 4)) || (hb && !aligned_to(p->dbias, 4))) return SS_ERR_ALIGN;
    if (q->rows > 0) {
        if (!s || !q->stats || !p->dout || !p->dx || (two && !p->dresidual)) return SS_ERR_NULL;
        if (!aligned_to(s, e.held) || !aligned_to(q->stats, 4) || !aligned_to(p->dout, e.io) || !aligned_to(p->dx, e.io) ||
            (res && !aligned_to(p->dsummed, e.held)) || (two && !aligned_to(p->dresidual, 4)))
            return SS_ERR_ALIGN;
        if (!p->workspace || p->workspace_bytes < ss_norm_workspace_bytes(q)) return SS_ERR_WORKSPACE;
        if (!aligned_to(p->workspace, 256)) return SS_ERR_ALIGN;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    ss::NormArgs a = norm_args(q);
    if (q->rows > 0) {
        a.s = s; a.dout = p->dout; a.dsummed = res ? p->dsummed : nullptr;
        a.dx = p->dx; a.dresidual = p->dresidual;
        a.mean = q->stats;
        a.rstd = q->stats + q->rows;
        a.part = static_cast<float*>(p->workspace);
        ss::norm_dispatch(a, q->io_dtype, q->flags, true, st);
    }
    if (hw || hb) {
        const int columns = (q->width + 31) / 32;
        const dim3 grid((unsigned)(columns < ss::NORM_MOST_WORKGROUPS ? columns : ss::NORM_MOST_WORKGROUPS), hb ? 2u : 1u);
        hipLaunchKernelGGL(ss::norm_parts_kernel, grid, dim3(1024), 0, st, a.part, hw ? p->dweight : nullptr,
                           hb ? p->dbias : nullptr, q->width, q->rows > 0 ? ss::norm_parts(q->rows, q->width) : 0);
    }
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
