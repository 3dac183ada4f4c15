// Products in 8-bit integers for gfx950: the quantiser of rows, and the product on the matrix cores, with the C-ABI
// entry points (see include/ss_quant.h).
//
// Products are C = A B^T with both operands contiguous along the contraction index, rows `pitch` bytes apart and the pitch a
// multiple of the 128 bytes that a step of the contraction takes, so no kernel has a tail along it.  Results whose rows
// are tokens take the tokens as A and the weight as B; results with the sequence last take the weight as A and one batch
// entry's tokens as B.
#include <hip/hip_runtime.h>
#include <type_traits>

#include "ss_quant.h"
#include "ss_slices.h"

namespace ss {

constexpr int Q_STEP = 128;                      // bytes of the contraction index that a step takes
constexpr float Q_LEAST = 7.52316384526264e-37f;  // 2^-120

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ---- the quantiser --------------------------------------------------------------------------------
// max |x| of a row, as the bits of a float: for magnitudes the order of the bits is that of the numbers, and infinities and NaN
// are above all of them.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
struct RowScale {
    float scale, inv;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top)
{
    RowScale r;
    const float m = __uint_as_float(top);
    if (top >= 0x7f800000u) {          // an infinity or NaN
        r.scale = __uint_as_float(0x7fc00000u);
        r.inv = 0.0f;
    } else if (m < Q_LEAST) {
        r.scale = 0.0f;
        r.inv = 0.0f;
    } else {
        r.scale = m / 127.0f;
        r.inv = 127.0f / m;
    }
    return r;
}
// round(v inv), ties to even; a value without a number (its row comes out as NaN) gives 0
__device__ __forceinline__ int quantised(float v, float inv)
{
    const float p = v * inv;
    return p == p ? (int)rintf(p) : 0;
}
__device__ __forceinline__ uint2 quantised8(const float (&v)[8], float inv)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[h] |= (uint32_t(quantised(v[4 * h + j], inv)) & 0xffu) << (8 * j);
    }
    return make_uint2(w[0], w[1]);
}

// Rows contiguous along dim: G lanes hold a row in registers, V slices of 8 each.
template <typename T, int G, int V>
__global__ __launch_bounds__(G > 256 ? G : 256) void quant_rows_kernel(const T* x, int8_t* q, float* scale, int rows, int dim, int pitch)
{
    constexpr int THREADS = G > 256 ? G : 256, SIDE = THREADS / G, WAVES = G > WAVE ? G / WAVE : 1;
    __shared__ uint32_t lds[WAVES];
    const int gl = threadIdx.x % G, last = (dim - 1) / 8 * 8;
    const int row0 = blockIdx.x * SIDE + threadIdx.x / G;
    const bool valid = row0 < rows;
    const int row = min(row0, rows - 1);
    const bool whole = dim % 8 == 0 || (dim >= 8 && row < rows - 1);
    const T* r = x + (int64_t)row * dim;
    typename io8<T>::raw raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = slice_load<T>(r, min((v * G + gl) * 8, last), dim, whole);
    float f[V][8];
    uint32_t top = 0u;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = dim - (v * G + gl) * 8;
        io8<T>::unpack(raw[v], f[v]);
        if (n < 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[v][j] = j < n ? f[v][j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(f[v][j]));
    }
#pragma unroll
    for (int s = 1; s < (G < WAVE ? G : WAVE); s *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if constexpr (G > WAVE) {
        if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, lds[w]);
    }
    const RowScale s = row_scale(top);
    if (!valid) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = (v * G + gl) * 8;
        if (at < pitch) *reinterpret_cast<uint2*>(q + (int64_t)row * pitch + at) = quantised8(f[v], s.inv);
    }
    if (gl == 0) scale[row] = s.scale;
}
// Rows that do not fit: a workgroup a row, read twice.
template <typename T>
__global__ __launch_bounds__(1024) void quant_rows_wide_kernel(const T* x, int8_t* q, float* scale, int dim, int pitch)
{
    __shared__ uint32_t lds[16];
    const T* r = x + (int64_t)blockIdx.x * dim;
    uint32_t top = 0u;
    for (int k = threadIdx.x; k < dim; k += 1024) top = max(top, magnitude(io_to_f32<T>(r[k])));
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) top = max(top, lds[w]);
    const RowScale s = row_scale(top);
    for (int k = threadIdx.x; k < pitch; k += 1024)
        q[(int64_t)blockIdx.x * pitch + k] = k < dim ? (int8_t)quantised(io_to_f32<T>(r[k]), s.inv) : (int8_t)0;
    if (threadIdx.x == 0) scale[blockIdx.x] = s.scale;
}

// Sequence last, x (batch, dim, L).  First the largest magnitudes of Q_CHUNK channels at a time, (chunks, batch L); ...
constexpr int Q_CHUNK = 128;
template <typename T>
__global__ __launch_bounds__(256) void quant_tops_kernel(const T* x, uint32_t* tops, int batch, int dim, int L)
{
    // thread: 8 tokens, every 8th channel of the chunk; 32 threads side by side
    __shared__ uint32_t lds[8][32][9];
    const int t0 = blockIdx.x * 256 + (threadIdx.x % 32) * 8, kk = threadIdx.x / 32, b = blockIdx.z, k0 = blockIdx.y * Q_CHUNK;
    const int last = (L - 1) / 8 * 8, at = min(t0, last);
    uint32_t top[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    for (int k = k0 + kk; k < min(k0 + Q_CHUNK, dim); k += 8) {
        const bool whole = L % 8 == 0 || (L >= 8 && !(b == batch - 1 && k == dim - 1));
        float v[8];
        io8<T>::unpack(slice_load<T>(x + ((int64_t)b * dim + k) * L, at, L, whole), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) top[j] = max(top[j], magnitude(v[j]));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[kk][threadIdx.x % 32][j] = top[j];
    __syncthreads();
    const int i = threadIdx.x / 8, j = threadIdx.x % 8, t = blockIdx.x * 256 + threadIdx.x;
    uint32_t m = 0u;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, lds[w][i][j]);
    if (t < L) tops[(int64_t)blockIdx.y * batch * L + (int64_t)b * L + t] = m;
}
// ... then tiles of 64 tokens and 128 channels, turned through LDS.
template <typename T>
__global__ __launch_bounds__(256) void quant_turn_kernel(const T* x, const uint32_t* tops, int8_t* q, float* scale, int batch, int dim, int L, int pitch, int chunks)
{
    __shared__ __align__(16) int8_t tile[64][Q_STEP + 16];
    __shared__ float inv[64];
    const int t0 = blockIdx.x * 64, k0 = blockIdx.y * Q_STEP, b = blockIdx.z;
    if (threadIdx.x < 64) {
        const int t = t0 + threadIdx.x;
        uint32_t m = 0u;
        if (t < L)
            for (int c = 0; c < chunks; ++c) m = max(m, tops[(int64_t)c * batch * L + (int64_t)b * L + t]);
        const RowScale s = row_scale(m);
        inv[threadIdx.x] = s.inv;
        if (blockIdx.y == 0 && t < L) scale[(int64_t)b * L + t] = s.scale;
    }
    __syncthreads();
    const int last = (L - 1) / 8 * 8, i = threadIdx.x % 8, at = min(t0 + 8 * i, last);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int kl = r * 32 + threadIdx.x / 8, k = k0 + kl;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (k < dim) {
            const bool whole = L % 8 == 0 || (L >= 8 && !(b == batch - 1 && k == dim - 1));
            io8<T>::unpack(slice_load<T>(x + ((int64_t)b * dim + k) * L, at, L, whole), v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[8 * i + j][kl] = (int8_t)quantised(v[j], inv[8 * i + j]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int tl = r * 32 + threadIdx.x / 8, t = t0 + tl;
        if (t < L)
            *reinterpret_cast<uint4*>(q + ((int64_t)b * L + t) * pitch + k0 + 16 * (threadIdx.x % 8)) =
                *reinterpret_cast<const uint4*>(&tile[tl][16 * (threadIdx.x % 8)]);
    }
}

// ---- the product -----------------------------------------------------------------------------------
struct QGemmArgs {
    int M, N, K;                       // K: bytes of a row, a multiple of Q_STEP
    const int8_t *A, *B;
    int64_t a_batch, b_batch;          // bytes
    const float *a_scale, *b_scale;
    int as_batch, bs_batch;            // elements
    const float *bias;                 // per row of A (bias_m) or row of B
    int bias_m;
    void* C;
    int64_t c_batch;                   // elements; rows N apart
};

// One workgroup: a tile of 128 x 128, 4 waves of 64 x 64 on v_mfma_i32_32x32x32_i8 (lane l supplies row l % 32 at the 16
// contraction indices from 16 (l / 32); accumulator element i of lane l is row 8 (i / 4) + 4 (l / 32) + i % 4, column l % 32).
// A step's 128 bytes of the tile's rows go straight from memory to LDS, in pieces of 16 bytes whose place in the row is the
// piece's number XOR the row's last three bits, so that the lanes of a read, which take one piece of 32 rows, spread over the banks.
template <typename T>
__global__ __launch_bounds__(256) void qgemm_kernel(QGemmArgs a)
{
    constexpr int TILE = 128;
    __shared__ __align__(16) int8_t lds[2][2][TILE * Q_STEP];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, b = blockIdx.z;
    const int m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
    const int8_t *A = a.A + b * a.a_batch, *B = a.B + b * a.b_batch;
    auto load = [&](int k0, int buf) {
        // 8 lanes a row, 8 rows a wave and request, 4 requests a wave and operand
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = (r * 4 + wave) * 8 + lane / 8, piece = (lane & 7) ^ (row & 7);
            const int8_t* pa = A + (int64_t)min(m0 + row, a.M - 1) * a.K + k0 + 16 * piece;
            const int8_t* pb = B + (int64_t)min(n0 + row, a.N - 1) * a.K + k0 + 16 * piece;
            int8_t* la = &lds[buf][0][(r * 4 + wave) * 8 * Q_STEP];
            int8_t* lb = &lds[buf][1][(r * 4 + wave) * 8 * Q_STEP];
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)pa, (__attribute__((address_space(3))) void*)la, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)pb, (__attribute__((address_space(3))) void*)lb, 16, 0, 0);
        }
    };
    const int wm = (wave / 2) * 64, wn = (wave % 2) * 64;
    i32x16 acc[2][2] = {};
    load(0, 0);
    for (int k0 = 0, buf = 0; k0 < a.K; k0 += Q_STEP, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's requests of the step have arrived in LDS
        __syncthreads();   // everybody's have, and the other buffer's have been read
        if (k0 + Q_STEP < a.K) load(k0 + Q_STEP, buf ^ 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            i32x4 fa[2], fb[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int ra = wm + 32 * t + lane % 32, rb = wn + 32 * t + lane % 32, piece = 2 * kk + lane / 32;
                fa[t] = *reinterpret_cast<const i32x4*>(&lds[buf][0][ra * Q_STEP + 16 * (piece ^ (ra & 7))]);
                fb[t] = *reinterpret_cast<const i32x4*>(&lds[buf][1][rb * Q_STEP + 16 * (piece ^ (rb & 7))]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }
    T* C = static_cast<T*>(a.C) + b * a.c_batch;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int n = n0 + wn + 32 * j + lane % 32;
        if (n >= a.N) continue;
        const float sn = a.b_scale[b * a.bs_batch + n], bn = a.bias && !a.bias_m ? a.bias[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int m = m0 + wm + 32 * i + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
                if (m >= a.M) continue;
                const float bm = a.bias && a.bias_m ? a.bias[m] : bn;
                C[(int64_t)m * a.N + n] = f32_to_io<T>(fmaf((float)acc[i][j][e], a.a_scale[b * a.as_batch + m] * sn, bm));
            }
    }
}

template <typename T>
void qgemm_launch(const QGemmArgs& a, int batch, hipStream_t st)
{
    hipLaunchKernelGGL(qgemm_kernel<T>, dim3((unsigned)((a.N + 127) / 128), (unsigned)((a.M + 127) / 128), (unsigned)batch), dim3(256), 0, st, a);
}

// ---- launches of the quantiser ------------------------------------------------------------------------
struct QuantSizes {
    int batch, L, dim, pitch;
    int chunks;   // of channels, sequence last
};
template <typename T>
void quant_launch(const QuantSizes& z, bool seq_last, const void* xv, int8_t* q, float* scale, uint32_t* tops, hipStream_t st)
{
    const T* x = static_cast<const T*>(xv);
    if (seq_last) {
        hipLaunchKernelGGL(quant_tops_kernel<T>, dim3((unsigned)((z.L + 255) / 256), (unsigned)z.chunks, (unsigned)z.batch), dim3(256), 0, st, x, tops, z.batch,
                           z.dim, z.L);
        hipLaunchKernelGGL(quant_turn_kernel<T>, dim3((unsigned)((z.L + 63) / 64), (unsigned)(z.pitch / Q_STEP), (unsigned)z.batch), dim3(256), 0, st, x, tops,
                           q, scale, z.batch, z.dim, z.L, z.pitch, z.chunks);
        return;
    }
    const int rows = z.batch * z.L;
    auto go = [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, V = decltype(v)::value, SIDE = (G > 256 ? G : 256) / G;
        hipLaunchKernelGGL((quant_rows_kernel<T, G, V>), dim3((unsigned)((rows + SIDE - 1) / SIDE)), dim3(G > 256 ? G : 256), 0, st, x, q, scale, rows, z.dim,
                           z.pitch);
    };
    typedef std::integral_constant<int, 1> one;
    typedef std::integral_constant<int, 2> two;
    typedef std::integral_constant<int, 4> four;
    if (z.pitch <= 512) go(std::integral_constant<int, 64>{}, one{});
    else if (z.pitch <= 2048 && rows >= 1024) {
        if (z.pitch <= 1024) go(std::integral_constant<int, 64>{}, two{});
        else go(std::integral_constant<int, 64>{}, four{});
    } else if (z.pitch <= 2048) go(std::integral_constant<int, 256>{}, one{});
    else if (z.pitch <= 4096) go(std::integral_constant<int, 256>{}, two{});
    else if (z.pitch <= 8192) go(std::integral_constant<int, 256>{}, four{});
    else if (z.pitch <= 16384) go(std::integral_constant<int, 1024>{}, two{});
    else hipLaunchKernelGGL(quant_rows_wide_kernel<T>, dim3((unsigned)rows), dim3(1024), 0, st, x, q, scale, z.dim, z.pitch);
}

}  // namespace ss

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

int check_sizes(int32_t batch, int32_t seqlen, int32_t dim, int32_t io_dtype)
{
    if (batch < 0 || seqlen < 0 || dim < 1) return SS_ERR_SHAPE;
    if (dim > SS_QUANT_MAX_DIM) return SS_ERR_UNSUPPORTED;
    if (io_dtype != SS_F32 && io_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if ((int64_t)batch * seqlen >= 0x7fffffffL - 65536) return SS_ERR_UNSUPPORTED;
    return SS_OK;
}
int chunks_of(int dim) { return (dim + ss::Q_CHUNK - 1) / ss::Q_CHUNK; }
size_t tops_bytes(int batch, int seqlen, int dim) { return round_up((size_t)chunks_of(dim) * batch * seqlen * sizeof(uint32_t), 256); }

void quantise(const ss::QuantSizes& z, bool seq_last, int io, const void* x, int8_t* q, float* scale, void* tops, hipStream_t st)
{
    if (io == SS_BF16) ss::quant_launch<ss::bf16_t>(z, seq_last, x, q, scale, static_cast<uint32_t*>(tops), st);
    else ss::quant_launch<float>(z, seq_last, x, q, scale, static_cast<uint32_t*>(tops), st);
}

// Scratch of a product: quantised tokens, their scales, and the maxima of tokens with the sequence last.
struct QSpace {
    size_t q, scale, tops, total;
};
QSpace q_space(const ss_qlinear_params* p)
{
    QSpace s{};
    if (p->flags & SS_Q_X_QUANTISED) return s;
    const size_t rows = (size_t)p->batch * p->seqlen;
    s.scale = round_up(rows * ss_quant_pitch(p->dim), 256);
    s.tops = s.scale + round_up(rows * sizeof(float), 256);
    s.total = s.tops + ((p->flags & SS_Q_X_SEQ_LAST) ? tops_bytes(p->batch, p->seqlen, p->dim) : 0);
    return s;
}

}  // namespace

extern "C" {

size_t ss_quant_pitch(int32_t dim) { return dim < 1 ? 0 : round_up((size_t)dim, ss::Q_STEP); }

size_t ss_quant_rows_scratch_bytes(const ss_quant_params* p)
{
    if (!p || p->batch < 0 || p->seqlen < 0 || p->dim < 1 || !(p->flags & SS_Q_X_SEQ_LAST)) return 0;
    return tops_bytes(p->batch, p->seqlen, p->dim);
}

int ss_quant_rows(const ss_quant_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const int rc = check_sizes(p->batch, p->seqlen, p->dim, p->io_dtype);
    if (rc != SS_OK) return rc;
    if (p->flags & ~(uint32_t)SS_Q_X_SEQ_LAST) return SS_ERR_UNSUPPORTED;
    if (p->batch == 0 || p->seqlen == 0) return SS_OK;
    const bool seq_last = p->flags & SS_Q_X_SEQ_LAST;
    if (seq_last && (p->batch > 65535 || chunks_of(p->dim) > 65535)) return SS_ERR_UNSUPPORTED;
    if (!p->x || !p->q || !p->scale) return SS_ERR_NULL;
    if (!aligned_to(p->x, p->io_dtype == SS_BF16 ? 2 : 4) || !aligned_to(p->q, 16) || !aligned_to(p->scale, 4)) return SS_ERR_ALIGN;
    const size_t need = ss_quant_rows_scratch_bytes(p);
    if (need && (!p->scratch || p->scratch_bytes < need)) return SS_ERR_WORKSPACE;
    if (need && !aligned_to(p->scratch, 256)) return SS_ERR_ALIGN;
    const ss::QuantSizes z = {p->batch, p->seqlen, p->dim, (int)ss_quant_pitch(p->dim), chunks_of(p->dim)};
    quantise(z, seq_last, p->io_dtype, p->x, static_cast<int8_t*>(p->q), p->scale, p->scratch, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

size_t ss_qlinear_scratch_bytes(const ss_qlinear_params* p)
{
    if (!p || p->batch < 0 || p->seqlen < 0 || p->dim < 1) return 0;
    return q_space(p).total;
}

int ss_qlinear(const ss_qlinear_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const int rc = check_sizes(p->batch, p->seqlen, p->dim, p->io_dtype);
    if (rc != SS_OK) return rc;
    if (p->features < 1) return SS_ERR_SHAPE;
    if (p->features > 0x7fffffff - 65536) return SS_ERR_UNSUPPORTED;
    if (p->flags & ~(uint32_t)(SS_Q_X_SEQ_LAST | SS_Q_OUT_SEQ_LAST | SS_Q_HAS_BIAS | SS_Q_X_QUANTISED)) return SS_ERR_UNSUPPORTED;
    const bool x_last = p->flags & SS_Q_X_SEQ_LAST, out_last = p->flags & SS_Q_OUT_SEQ_LAST, done = p->flags & SS_Q_X_QUANTISED, hb = p->flags & SS_Q_HAS_BIAS;
    if (x_last && done) return SS_ERR_UNSUPPORTED;
    if (p->batch == 0 || p->seqlen == 0) return SS_OK;
    if ((x_last || out_last) && p->batch > 65535) return SS_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)p->batch * p->seqlen;
    // tiles of the grid's second and third axes
    if (x_last && chunks_of(p->dim) > 65535) return SS_ERR_UNSUPPORTED;
    if ((out_last ? (int64_t)p->features : rows) > (int64_t)65535 * 128) return SS_ERR_UNSUPPORTED;
    if (!p->x || !p->weight || !p->scale || !p->out || (done && !p->x_scale) || (hb && !p->bias)) return SS_ERR_NULL;
    const size_t esz = p->io_dtype == SS_BF16 ? 2 : 4;
    if (!aligned_to(p->x, done ? 16 : esz) || !aligned_to(p->weight, 16) || !aligned_to(p->scale, 4) || !aligned_to(p->out, esz) ||
        (done && !aligned_to(p->x_scale, 4)) || (hb && !aligned_to(p->bias, 4)))
        return SS_ERR_ALIGN;
    const QSpace s = q_space(p);
    char* const ws = static_cast<char*>(p->scratch);
    if (s.total && (!ws || p->scratch_bytes < s.total)) return SS_ERR_WORKSPACE;
    if (s.total && !aligned_to(ws, 256)) return SS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int pitch = (int)ss_quant_pitch(p->dim);
    const int8_t* q = static_cast<const int8_t*>(p->x);
    const float* q_scale = p->x_scale;
    if (!done) {
        const ss::QuantSizes z = {p->batch, p->seqlen, p->dim, pitch, chunks_of(p->dim)};
        quantise(z, x_last, p->io_dtype, p->x, reinterpret_cast<int8_t*>(ws + s.q), reinterpret_cast<float*>(ws + s.scale), ws + s.tops, st);
        q = reinterpret_cast<const int8_t*>(ws + s.q);
        q_scale = reinterpret_cast<const float*>(ws + s.scale);
    }
    ss::QGemmArgs g{};
    g.K = pitch;
    g.bias = hb ? p->bias : nullptr;
    g.C = p->out;
    const int8_t* w = static_cast<const int8_t*>(p->weight);
    int batch = 1;
    if (out_last) {
        g.M = p->features; g.N = p->seqlen;
        g.A = w; g.a_scale = p->scale;
        g.B = q; g.b_scale = q_scale;
        g.b_batch = (int64_t)p->seqlen * pitch;
        g.bs_batch = p->seqlen;
        g.c_batch = (int64_t)p->features * p->seqlen;
        g.bias_m = 1;
        batch = p->batch;
    } else {
        g.M = (int)rows; g.N = p->features;
        g.A = q; g.a_scale = q_scale;
        g.B = w; g.b_scale = p->scale;
    }
    if (p->io_dtype == SS_BF16) ss::qgemm_launch<ss::bf16_t>(g, batch, st);
    else ss::qgemm_launch<float>(g, batch, st);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
