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
constexpr int64_t MOST_THREADS = 0x7fffffff;      // of a launch (its limit is 2^32)
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
        r.inv = 127.0f * (1.0f / m);
    }
    return r;
}
// round(v inv) of four values, ties to even, as the bytes of a word: 1.5 2^23 added to the rounded product leaves the whole number in the
// low byte.  inv is 0 in rows that come out as zeros or NaN; their bytes are 0 whatever stands in them.
__device__ __forceinline__ uint32_t quantised4(float v0, float v1, float v2, float v3, float inv)
{
#pragma clang fp contract(off)
    constexpr float up = 12582912.0f;
    const float p0 = v0 * inv, p1 = v1 * inv, p2 = v2 * inv, p3 = v3 * inv;
    const uint32_t low = __builtin_amdgcn_perm(__float_as_uint(p1 + up), __float_as_uint(p0 + up), 0x0c0c0400u);
    const uint32_t high = __builtin_amdgcn_perm(__float_as_uint(p3 + up), __float_as_uint(p2 + up), 0x04000c0cu);
    return inv == 0.0f ? 0u : low | high;
}
__device__ __forceinline__ uint2 quantised8(const float (&v)[8], float inv)
{
    return make_uint2(quantised4(v[0], v[1], v[2], v[3], inv), quantised4(v[4], v[5], v[6], v[7], inv));
}

// Rows contiguous along dim: G lanes hold a row in registers, V slices of 8 each, so it is read once.  Bound by HBM: 16384 x 2048 bf16
// (67 MB in, 34 MB out) 24 us when not in a cache, 4.2 TB/s.
template <typename T, int G, int V>
__global__ __launch_bounds__(G > 256 ? G : 256) void quant_rows_kernel(const T* x, int8_t* q, float* scale, int rows, int dim, int pitch)
{
    constexpr int THREADS = G > 256 ? G : 256, SIDE = THREADS / G, WAVES = G > WAVE ? G / WAVE : 1;
    __shared__ uint32_t lds[WAVES];
    const int gl = threadIdx.x % G;
    const int row0 = blockIdx.x * SIDE + threadIdx.x / G;
    const bool valid = row0 < rows;
    const int row = min(row0, rows - 1);
    const bool whole = slice_whole(dim, row == rows - 1);
    const int limit = slice_limit(dim, whole);
    const T* r = x + (int64_t)row * dim;
    typename io8<T>::raw raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = slice_request<T, G == 64 && V == 1>(r, (v * G + gl) * 8, dim, limit);
    if (!whole) {
#pragma unroll
        for (int v = 0; v < V; ++v) slice_settle<T>(raw[v], (v * G + gl) * 8, dim, limit, false);
    }
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
// Rows that do not fit: a workgroup a row, read twice, the second time from the caches.  An element a thread and access, which
// is what bounds it: 2048 x 20000 bf16 (123 MB) 57 us, 2.2 TB/s; kept simple, as rows this wide are few.
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
        q[(int64_t)blockIdx.x * pitch + k] = k < dim ? (int8_t)quantised4(io_to_f32<T>(r[k]), 0.0f, 0.0f, 0.0f, s.inv) : (int8_t)0;
    if (threadIdx.x == 0) scale[blockIdx.x] = s.scale;
}

// Slices of eight tokens with the sequence last, x (batch, dim, L): of channel k, the last one's for those past it, ...
template <typename T>
__device__ __forceinline__ typename io8<T>::raw request_channel(const T* x, int b, bool last_entry, int k, int dim, int t0, int L)
{
    const int kk = min(k, dim - 1);
    return slice_request<T, true>(x + ((int64_t)b * dim + kk) * L, t0, L, slice_limit(L, slice_whole(L, last_entry && kk == dim - 1)));
}
// ... and of four channels as floats, zeros for those past the last.
template <typename T>
__device__ __forceinline__ void settle4(typename io8<T>::raw (&raw)[4], bool last_entry, int k0, int dim, int t0, int L, float (&v)[4][8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool whole = slice_whole(L, last_entry && k0 + e >= dim - 1);
        slice_settle<T>(raw[e], t0, L, slice_limit(L, whole), whole);
        io8<T>::unpack(raw[e], v[e]);
        if (k0 + e >= dim)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[e][j] = 0.0f;
    }
}
// In two launches, where registers do not hold the channels.  First the largest magnitudes of Q_CHUNK channels at a time, (chunks, batch L); ...
// (2 x 8192 x 4096 bf16, 134 MB, 30 us)
constexpr int Q_CHUNK = 128;
template <typename T>
__global__ __launch_bounds__(256) void quant_tops_kernel(const T* x, uint32_t* tops, int batch, int dim, int L)
{
    // thread: 8 tokens, every 8th channel of the chunk; 32 threads side by side
    __shared__ uint32_t lds[8][32][9];
    const int t0 = blockIdx.x * 256 + (threadIdx.x % 32) * 8, kk = threadIdx.x / 32, b = blockIdx.z, k0 = blockIdx.y * Q_CHUNK;
    uint32_t top[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    for (int k = k0 + kk; k < min(k0 + Q_CHUNK, dim); k += 8) {
        const bool whole = slice_whole(L, b == batch - 1 && k == dim - 1);
        const int limit = slice_limit(L, whole);
        typename io8<T>::raw r = slice_request<T, true>(x + ((int64_t)b * dim + k) * L, t0, L, limit);
        slice_settle<T>(r, t0, L, limit, whole);
        float v[8];
        io8<T>::unpack(r, v);
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
// ... then tiles of 128 tokens and 128 channels, turned through LDS: a thread takes 8 tokens of four channels and puts each token's four
// bytes down as a word; rows of 132 bytes spread those of a wave over all banks.  2 x 8192 x 4096 bf16 35 us, 5.8 TB/s (64 tokens, bytes put down one
// by one: 1.8 times as long).
constexpr int TURN_TOKENS = 128;
template <typename T>
__global__ __launch_bounds__(256) void quant_turn_kernel(const T* x, const uint32_t* tops, int8_t* q, float* scale, int batch, int dim, int L, int pitch, int chunks)
{
    constexpr int ROW = Q_STEP / 4 + 1;   // words
    __shared__ uint32_t tile[TURN_TOKENS * ROW];
    __shared__ uint32_t half[2][TURN_TOKENS];
    __shared__ float inv[TURN_TOKENS];
    const int t0 = blockIdx.x * TURN_TOKENS, k0 = blockIdx.y * Q_STEP, b = blockIdx.z;
    {
        const int t = threadIdx.x % TURN_TOKENS, h = threadIdx.x / TURN_TOKENS;
        uint32_t m = 0u;
        if (t0 + t < L) {
            const uint32_t* p = tops + (int64_t)b * L + t0 + t;
#pragma unroll 8
            for (int c = h; c < chunks; c += 2) m = max(m, p[(int64_t)c * batch * L]);
        }
        half[h][t] = m;
    }
    // the channels' values are requested before anything waits for the scales
    const int i = threadIdx.x % 16, kq = threadIdx.x / 16;   // tokens 8 i .., channels 4 kq .. of 64
    typename io8<T>::raw raw[2][4];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[r][e] = request_channel<T>(x, b, b == batch - 1, k0 + 64 * r + 4 * kq + e, dim, t0 + 8 * i, L);
    __syncthreads();
    if (threadIdx.x < TURN_TOKENS) {
        const RowScale s = row_scale(max(half[0][threadIdx.x], half[1][threadIdx.x]));
        inv[threadIdx.x] = s.inv;
        if (blockIdx.y == 0 && t0 + (int)threadIdx.x < L) scale[(int64_t)b * L + t0 + threadIdx.x] = s.scale;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float v[4][8];
        settle4<T>(raw[r], b == batch - 1, k0 + 64 * r + 4 * kq, dim, t0 + 8 * i, L, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[(8 * i + j) * ROW + 16 * r + kq] = quantised4(v[0][j], v[1][j], v[2][j], v[3][j], inv[8 * i + j]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < TURN_TOKENS / 32; ++r) {
        const int tl = r * 32 + threadIdx.x / 8, t = t0 + tl, c = threadIdx.x % 8;
        if (t < L) {
            const uint32_t* p = &tile[tl * ROW + 4 * c];
            *reinterpret_cast<uint4*>(q + ((int64_t)b * L + t) * pitch + k0 + 16 * c) = make_uint4(p[0], p[1], p[2], p[3]);
        }
    }
}

// The largest magnitudes of eight values each lane has seen, and their exchange over LDS: 16-bit ones in pairs.
template <typename T>
struct Tops {
    uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
    __device__ __forceinline__ void see(const typename io8<T>::raw& r)
    {
        float v[8];
        io8<T>::unpack(r, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = max(w[j], magnitude(v[j]));
    }
    static __device__ __forceinline__ void put(uint32_t* to, int i, uint32_t v) { to[i] = v; }
};
template <>
struct Tops<bf16_t> {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    static constexpr int N = 4;
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    __device__ __forceinline__ void see(const io8<bf16_t>::raw& r)
    {
        const uint32_t v[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = larger(w[j], v[j] & 0x7fff7fffu);
    }
    static __device__ __forceinline__ void put(uint32_t* to, int i, uint32_t v)
    {
        to[2 * i] = v << 16;
        to[2 * i + 1] = v & 0xffff0000u;
    }
};

// Where a workgroup's registers hold all channels of 8 WIDE tokens, one pass: a thread has 8 tokens of four channels R times, the tokens' scales
// come from an exchange over the workgroup, and a thread's four bytes of a token are a word of its row, of which a wave writes
// whole lines.  Bound by the pieces in which rows are read, 16 WIDE bytes of bf16: 4 x 4096 x 1531 bf16 (50 MB in, 25 MB out) takes 18 us at
// 64 bytes (4.2 TB/s); a call of it 23 at 64, 32 at 32, and 32 in two launches.  Up to 64 registers a thread where they do without spilling, so that two
// workgroups of 1024 share a unit.
template <typename T, int THREADS, int WIDE, int R>
__global__ __launch_bounds__(THREADS, R * sizeof(T) <= 4 && THREADS * R < 2048 * WIDE ? 8 : 4) void quant_held_kernel(const T* x, int8_t* q, float* scale, int batch, int dim, int L, int pitch, int tiles)
{
    constexpr int WAVES = THREADS / WAVE, TOKENS = 8 * WIDE, SIDE = THREADS / WIDE;
    __shared__ uint32_t lds[WAVES][TOKENS];
    __shared__ float inv[TOKENS];
    // the XCDs get neighbouring tiles, which share lines
    const int share = gridDim.x / 8, id = blockIdx.x < 8 * share ? (blockIdx.x % 8) * share + blockIdx.x / 8 : blockIdx.x;
    const int b = id / tiles, t0 = (id - b * tiles) * TOKENS, i = threadIdx.x % WIDE, kq = 4 * (threadIdx.x / WIDE);
    const bool last = b == batch - 1;
    typename io8<T>::raw raw[R][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[r][e] = request_channel<T>(x, b, last, r * 4 * SIDE + kq + e, dim, t0 + 8 * i, L);
    Tops<T> top;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool whole = slice_whole(L, last && r * 4 * SIDE + kq + e >= dim - 1);
            slice_settle<T>(raw[r][e], t0 + 8 * i, L, slice_limit(L, whole), whole);
            top.see(raw[r][e]);
        }
    // lanes of the same tokens halve the words between them, then take the larger
    int word = 0, lanes = WIDE;
#pragma unroll
    for (int n = Tops<T>::N / 2; n >= 1; n /= 2, lanes *= 2) {
        const bool up = threadIdx.x & lanes;
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const uint32_t mine = up ? top.w[j + n] : top.w[j], other = up ? top.w[j] : top.w[j + n];
            top.w[j] = Tops<T>::larger(mine, (uint32_t)__shfl_xor((int)other, lanes));
        }
        word += up ? n : 0;
    }
#pragma unroll
    for (; lanes < WAVE; lanes *= 2) top.w[0] = Tops<T>::larger(top.w[0], (uint32_t)__shfl_xor((int)top.w[0], lanes));
    if (threadIdx.x % WAVE < WIDE * Tops<T>::N) Tops<T>::put(&lds[threadIdx.x / WAVE][8 * i], word, top.w[0]);
    __syncthreads();
    if (threadIdx.x < TOKENS) {
        uint32_t m = 0u;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = max(m, lds[w][threadIdx.x]);
        const RowScale s = row_scale(m);
        inv[threadIdx.x] = s.inv;
        if (t0 + (int)threadIdx.x < L) scale[(int64_t)b * L + t0 + threadIdx.x] = s.scale;
    }
    __syncthreads();
    int8_t* const to = q + ((int64_t)b * L + t0 + 8 * i) * pitch;
    float by[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) by[j] = inv[8 * i + j];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int k = r * 4 * SIDE + kq;
        if (k >= pitch) break;
        float v[4][8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            io8<T>::unpack(raw[r][e], v[e]);
            if (k + e >= dim)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[e][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (t0 + 8 * i + j < L) *reinterpret_cast<uint32_t*>(to + (int64_t)j * pitch + k) = quantised4(v[0][j], v[1][j], v[2][j], v[3][j], by[j]);
    }
}

// ---- the product -----------------------------------------------------------------------------------
struct QGemmArgs {
    int M, N, K, batch;                // K: bytes of a row, a multiple of Q_STEP
    const int8_t *A, *B;
    int64_t a_batch, b_batch;          // bytes
    const float *a_scale, *b_scale;
    int as_batch, bs_batch;            // elements
    const float *bias;                 // per row of A (bias_m) or row of B
    int bias_m;
    void* C;
    int64_t c_batch;                   // elements; rows N apart
};

// Tiles of BM x BN by WM x WN waves, each TM x TN products of v_mfma_i32_32x32x32_i8 (lane l supplies row l % 32 of an operand at
// the 16 contraction indices from 16 (l / 32); accumulator element e of lane l is row 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32).
// B's rows are the instruction's rows, so that a lane holds four neighbours of a row of C.
//
// A step's 128 bytes of the tile's rows go straight from memory to LDS, STAGES - 1 steps ahead, in pieces of 16 bytes whose place in the
// row is the piece's number XOR the row's last three bits, so that the lanes of a read, which take one piece of 32 rows, spread
// over the banks.  Results are turned through a strip of LDS that each wave has to itself and leave in whole lines.
//
// What bounds it: with all units at work the clock, which the matrix cores' power sets: 8192 x 16384 x 2048 takes 295 us (1860
// TOP/s), 16384 x 2048 x 4096 133 us (2060; the library's 8-bit product reaches 1981 at 8192^3, the matrix cores by
// themselves, on constants, 4300).  A workgroup alone takes 1.13 us a step: 256 x 256 x 128 products are 0.87 us at the peak, its 8
// waves of 64 x 128 read 192 KB of LDS, which is as long again, beside them.  What each part brought at 8192 x 16384 x 2048: 128 x 128
// tiles 425 us, 256 x 256 342, turned results 322, staying for the next tile, whose first step is requested before this one's
// results are stored (PERSISTENT), 310, requests through buffer resources 304 (behind global ones the compiler waits for all
// LDS reads at once, as it counts such requests among them), requests between the products 295.
// bytes of a wave's strip: 32 rows of 32 results; 16-bit rows are set 16 bytes apart, 32-bit ones swizzled like the tiles
template <typename T> constexpr int strip_pitch() { return sizeof(T) == 2 ? 80 : 128; }

template <typename T, int WM, int WN, int TM, int TN, int STAGES, bool PERSISTENT>
__global__ __launch_bounds__(WM* WN* WAVE) void qgemm_kernel(QGemmArgs a)
{
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, WAVES = WM * WN, RA = BM / 8 / WAVES, RB = BN / 8 / WAVES;
    constexpr int PITCH = strip_pitch<T>(), STRIP = 32 * PITCH, STAGE = (BM + BN) * Q_STEP;
    static_assert(!PERSISTENT || STAGES == 2, "a tile's last step requests the next one's first step alone");
    __shared__ __align__(16) int8_t lds[STAGES * STAGE + WAVES * STRIP];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int nm = (a.M + BM - 1) / BM, nn = (a.N + BN - 1) / BN, tiles = nm * nn;
    const int64_t total = (int64_t)tiles * a.batch;
    const int wm = (wave / WN) * TM * 32, wn = (wave % WN) * TN * 32;
    int8_t* const strip = lds + STAGES * STAGE + wave * STRIP;
    rsrc_t ra, rb;   // the tile's rows of both operands, and where in them a lane reads
    uint32_t oa[RA], ob[RB];
    int m0, n0, b;
    // Where tile `id` lies: the XCDs get contiguous shares, and within one eight tiles of M are taken for each of N, so that what
    // is worked on at a time shares rows of both operands.
    auto place = [&](int64_t id) {
        if (total % 8 == 0) id = (id % 8) * (total / 8) + id / 8;
        b = (int)(id / tiles);
        const int t = (int)(id - (int64_t)b * tiles), group = t / (8 * nn), first = group * 8, size = min(nm - first, 8), in = t - group * 8 * nn;
        m0 = (first + in % size) * BM;
        n0 = in / size * BN;
        ra = make_rsrc(a.A + b * a.a_batch + (int64_t)m0 * a.K, (uint32_t)BM * (uint32_t)a.K);
        rb = make_rsrc(a.B + b * a.b_batch + (int64_t)n0 * a.K, (uint32_t)BN * (uint32_t)a.K);
        // 8 lanes a row, 8 rows a wave and request; rows past the end read the last one
#pragma unroll
        for (int r = 0; r < RA; ++r) {
            const int row = (r * WAVES + wave) * 8 + lane / 8;
            oa[r] = (uint32_t)min(row, a.M - 1 - m0) * (uint32_t)a.K + 16 * ((lane & 7) ^ (row & 7));
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int row = (r * WAVES + wave) * 8 + lane / 8;
            ob[r] = (uint32_t)min(row, a.N - 1 - n0) * (uint32_t)a.K + 16 * ((lane & 7) ^ (row & 7));
        }
    };
    // requests [from, to) of the RA + RB of a step
    auto load = [&](int k0, int buf, int from, int to) {
        int8_t* const l = lds + buf * STAGE + wave * 8 * Q_STEP;
#pragma unroll
        for (int r = 0; r < RA + RB; ++r)
            if (r >= from && r < to)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r < RA ? ra : rb, (__attribute__((address_space(3))) void*)(l + (r < RA ? 0 : BM - RA * WAVES * 8) * Q_STEP + r * WAVES * 8 * Q_STEP),
                                                         16, (int)(r < RA ? oa[r < RA ? r : 0] : ob[r < RA ? 0 : r - RA]), k0, 0, 0);
    };
    int64_t id = blockIdx.x;
    int buf = 0;   // of the step at hand; the step before lay in the buffer that the one STAGES - 1 later gets
    place(id);
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
        if (k == 0 || k * Q_STEP < a.K) load(k * Q_STEP, k, 0, RA + RB);
    for (;;) {
        const int64_t next = id + gridDim.x;
        const bool more = PERSISTENT && next < total;
        const int cm = m0 + wm, cn = n0 + wn, cb = b;
        i32x16 acc[TM][TN] = {};
        for (int k0 = 0; k0 < a.K; k0 += Q_STEP, buf = buf + 1 == STAGES ? 0 : buf + 1) {
            // this wave's requests of the step have arrived in LDS: all but those of the steps behind it that are under way
            if (STAGES > 2 && k0 + (STAGES - 2) * Q_STEP < a.K) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * (RA + RB)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            // everybody's have, and the buffer of the step before has been read (__syncthreads would wait for all requests)
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int ahead = buf == 0 ? STAGES - 1 : buf - 1;
            int k_ahead = k0 + (STAGES - 1) * Q_STEP;
            bool request = k_ahead < a.K;
            if (!request && more) {
                place(next);
                k_ahead = 0;
                request = true;
            }
            const int8_t* const from = lds + buf * STAGE;
            // The operands of AT of the step's four products a tile are read together: one by one their latency (about 130 clocks, four times a
            // step) is all that a wave of few tiles sees.
            constexpr int AT = TM * TN <= 4 ? 4 : 1;
#pragma unroll
            for (int k4 = 0; k4 < Q_STEP / 32; k4 += AT) {
                i32x4 fa[AT][TM], fb[AT][TN];
#pragma unroll
                for (int kk = 0; kk < AT; ++kk) {
                    const int piece = 2 * (k4 + kk) + lane / 32;
#pragma unroll
                    for (int t = 0; t < TM; ++t) {
                        const int r = wm + 32 * t + lane % 32;
                        fa[kk][t] = *reinterpret_cast<const i32x4*>(from + r * Q_STEP + 16 * (piece ^ (r & 7)));
                    }
#pragma unroll
                    for (int t = 0; t < TN; ++t) {
                        const int r = wn + 32 * t + lane % 32;
                        fb[kk][t] = *reinterpret_cast<const i32x4*>(from + BM * Q_STEP + r * Q_STEP + 16 * (piece ^ (r & 7)));
                    }
                }
                // The next step's requests go out between the products: in one go they would hold the wave up for as long as the
                // products take.
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kk = 0; kk < AT; ++kk) {
                    if (request) load(k_ahead, ahead, (RA + RB) * (k4 + kk) / 4, (RA + RB) * (k4 + kk + 1) / 4);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        T* const C = static_cast<T*>(a.C) + cb * a.c_batch;
        const float *sa = a.a_scale + cb * a.as_batch, *sb = a.b_scale + cb * a.bs_batch;
        float ms[TM], mb[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int m = min(cm + 32 * i + lane % 32, a.M - 1);
            ms[i] = sa[m];
            mb[i] = a.bias && a.bias_m ? a.bias[m] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            float ns[16], nb[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int n = min(cn + 32 * j + 8 * (e / 4) + 4 * (lane / 32) + e % 4, a.N - 1);
                ns[e] = sb[n];
                nb[e] = a.bias && !a.bias_m ? a.bias[n] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = fmaf((float)acc[i][j][e], ms[i] * ns[e], mb[i] + nb[e]);
                const int r = lane % 32;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (sizeof(T) == 2) {
                        *reinterpret_cast<uint2*>(strip + r * PITCH + 16 * q + 8 * (lane / 32)) =
                            make_uint2(pack_bf16x2(v[4 * q], v[4 * q + 1]), pack_bf16x2(v[4 * q + 2], v[4 * q + 3]));
                    } else {
                        *reinterpret_cast<float4*>(strip + r * PITCH + 16 * ((2 * q + lane / 32) ^ (r & 7))) =
                            make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                    }
                }
                // the strip is this wave's: its LDS accesses are carried out in order
                __builtin_amdgcn_wave_barrier();
                constexpr int E = 16 / sizeof(T), LANES = 32 / E;   // results a lane stores at a time, lanes of a row
#pragma unroll
                for (int h = 0; h < 32 * LANES / WAVE; ++h) {
                    const int row = h * (WAVE / LANES) + lane / LANES, c = lane % LANES;
                    const u32x4 w = *reinterpret_cast<const u32x4*>(strip + row * PITCH + 16 * (sizeof(T) == 2 ? c : c ^ (row & 7)));
                    const int m = cm + 32 * i + row, n = cn + 32 * j + E * c;
                    if (m < a.M && n < a.N) {
                        T* const to = C + (int64_t)m * a.N + n;
                        if (n + E <= a.N) {
                            if constexpr (sizeof(T) == 2) store_row16(to, w);
                            else store_any(to, 0u, w);
                        } else {
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (n + e < a.N) {
                                    if constexpr (sizeof(T) == 2) to[e] = bf16_t(w[e / 2] >> (16 * (e % 2)));
                                    else to[e] = __uint_as_float(w[e]);
                                }
                        }
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (!more) break;
        id = next;
    }
}

// ---- few tokens ----------------------------------------------------------------------------------------
// Up to 32 tokens: the weight's bytes bound it, so they go from memory to registers as operands, once each.  A workgroup takes 16
// of the weight's rows, its waves share the contraction index out in turn (units of Q_STEP), and their sums, integers, are
// added up through LDS.  v_mfma_i32_16x16x64_i8: lane l supplies row l % 16 (of the weight; a token of the other operand) at the 16
// indices from 16 (l / 16), so a request takes 64 bytes of each of 16 rows; element e of lane l is row 4 (l / 16) + e, token l % 16.
//
// FUSED: every workgroup brings the tokens to 8 bits itself, from registers into LDS, while its first weights are under way (one
// launch instead of two).
struct QFewArgs {
    int tokens, features, dim, pitch;
    const void* x;                   // FUSED: (tokens, dim) io values
    const int8_t* q;                 // else (tokens, pitch) and their scales
    const float* q_scale;
    const int8_t* w;
    const float *scale, *bias;
    void* out;                       // (tokens, features)
};
constexpr int FEW_SLICES = 4;        // most slices of 8 values of a thread, over all tokens, that a workgroup quantises itself
constexpr int FEW_AHEAD = 4;         // units of a wave whose weights are requested together

// Slices of 8 values that a token is dealt out in: whole waves of them, so that a wave's are of one token
__host__ __device__ __forceinline__ int few_slices(int pitch) { return (pitch / 8 + WAVE - 1) / WAVE * WAVE; }

template <typename T, int GROUPS, int WAVES, int SLICES>   // GROUPS of 16 tokens; SLICES of a thread where FUSED, else 0
__global__ __launch_bounds__(WAVES* WAVE) void qfew_kernel(QFewArgs a)
{
    constexpr int THREADS = WAVES * WAVE;
    constexpr bool FUSED = SLICES > 0;
    __shared__ __align__(16) int8_t lq[FUSED ? SLICES * THREADS * 8 : 16];
    __shared__ uint32_t tops[16];
    __shared__ float scales[GROUPS * 16];
    __shared__ __align__(16) i32x4 sums[WAVES][GROUPS][WAVE];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int n0 = blockIdx.x * 16, units = a.pitch / Q_STEP;
    const int8_t* const w = a.w + (int64_t)min(n0 + lane % 16, a.features - 1) * a.pitch + 16 * (lane / 16);
    [[maybe_unused]] typename io8<T>::raw raw[FUSED ? SLICES : 1];
    const int per = few_slices(a.pitch);
    if constexpr (FUSED) {
        if (threadIdx.x < 16) tops[threadIdx.x] = 0u;
#pragma unroll
        for (int v = 0; v < SLICES; ++v) {
            const int s = v * THREADS + threadIdx.x, t = min(s / per, a.tokens - 1), at = (s - s / per * per) * 8;
            raw[v] = slice_request<T, false>(static_cast<const T*>(a.x) + (int64_t)t * a.dim, at, a.dim, slice_limit(a.dim, slice_whole(a.dim, t == a.tokens - 1)));
        }
    }
    i32x4 fw[FEW_AHEAD][2];
    auto load = [&](int u0) {
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k) {
            const int64_t at = (int64_t)min(u0 + k * WAVES, units - 1) * Q_STEP;   // past the end: the last unit again, not used
            fw[k][0] = *reinterpret_cast<const i32x4*>(w + at);
            fw[k][1] = *reinterpret_cast<const i32x4*>(w + at + 64);
        }
    };
    load(wave);
    if constexpr (FUSED) {
        float f[SLICES][8];
        __syncthreads();
#pragma unroll
        for (int v = 0; v < SLICES; ++v) {
            const int s = v * THREADS + threadIdx.x, t = s / per, n = a.dim - (s - t * per) * 8;
            if (!slice_whole(a.dim, t >= a.tokens - 1)) slice_settle<T>(raw[v], a.dim - n, a.dim, slice_limit(a.dim, false), false);
            io8<T>::unpack(raw[v], f[v]);
            uint32_t top = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[v][j] = j < n ? f[v][j] : 0.0f;
                top = max(top, magnitude(f[v][j]));
            }
#pragma unroll
            for (int k = 1; k < WAVE; k *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, k));
            if (lane == 0 && t < a.tokens) atomicMax(&tops[t], top);
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < SLICES; ++v) {
            const int s = v * THREADS + threadIdx.x, t = s / per;
            const int at = (s - t * per) * 8;
            if (t < a.tokens && at < a.pitch) *reinterpret_cast<uint2*>(lq + t * a.pitch + at) = quantised8(f[v], row_scale(tops[t]).inv);
        }
        if (threadIdx.x < 16) scales[threadIdx.x] = row_scale(tops[threadIdx.x]).scale;
        __syncthreads();
    } else {
        for (int t = threadIdx.x; t < GROUPS * 16; t += THREADS) scales[t] = a.q_scale[min(t, a.tokens - 1)];
    }
    i32x4 acc[GROUPS] = {};
    for (int u0 = wave; u0 < units; u0 += FEW_AHEAD * WAVES) {
        i32x4 cur[FEW_AHEAD][2];
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k) {
            cur[k][0] = fw[k][0];
            cur[k][1] = fw[k][1];
        }
        if (u0 + FEW_AHEAD * WAVES < units) load(u0 + FEW_AHEAD * WAVES);
#pragma unroll
        for (int k = 0; k < FEW_AHEAD; ++k) {
            if (u0 + k * WAVES >= units) break;
            const int at = (u0 + k * WAVES) * Q_STEP + 16 * (lane / 16);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int t = min(16 * g + lane % 16, a.tokens - 1);
                i32x4 t0, t1;
                if constexpr (FUSED) {
                    t0 = *reinterpret_cast<const i32x4*>(lq + t * a.pitch + at);
                    t1 = *reinterpret_cast<const i32x4*>(lq + t * a.pitch + at + 64);
                } else {
                    const int8_t* q = a.q + (int64_t)t * a.pitch + at;
                    t0 = *reinterpret_cast<const i32x4*>(q);
                    t1 = *reinterpret_cast<const i32x4*>(q + 64);
                }
                acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cur[k][0], t0, acc[g], 0, 0, 0);
                acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cur[k][1], t1, acc[g], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) sums[wave][g][lane] = acc[g];
    __syncthreads();
    for (int i = threadIdx.x; i < GROUPS * WAVE; i += THREADS) {
        const int g = i / WAVE, l = i % WAVE, t = 16 * g + l % 16, n = n0 + 4 * (l / 16);
        i32x4 v = sums[0][g][l];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) v += sums[k][g][l];
        if (t >= a.tokens) continue;
        T* const to = static_cast<T*>(a.out) + (int64_t)t * a.features + n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.features) to[e] = f32_to_io<T>(fmaf((float)v[e], scales[t] * a.scale[n + e], a.bias ? a.bias[n + e] : 0.0f));
    }
}

// Where the tiles begin to pay: 33 tokens, weights and tokens not in a cache, the quantiser's launch included, would take here (four groups
// of 16) / take in tiles of 64 (us) 13.4 / 11.9 at 2048 x 8192, 14.3 / 16.1 at 4096 x 2048, 8.1 / 7.4 at 768 x 3008, 9.5 / 9.4 at 1500 x 700.
constexpr int FEW_TOKENS = 32;
// Waves of a workgroup: enough to fill the chip with (8 to a compute unit), while each has a unit.  us with 4 / 8 / 16 of them, weights
// and tokens not in a cache, one token and 16: 2048 x 8192 (dim x features) 6.2 7.8 13.1 and 10.3 11.6 15.9, 768 x 16384 7.5 12.6 23.2 and 11.5
// 15.5 26.4, 768 x 3008 4.0 4.9 6.8 and 7.0 7.5 8.0, 2560 x 5120 7.6 7.5 12.9 and 12.3 12.3 16.5, 5120 x 2560 8.5 8.5 7.7 and 12.9 12.3 12.5.  The
// lines between them are rough: fewer are ahead at 4096 x 2048 (6.5 5.7 7.4 and 10.7 9.6 11.5, 16 are taken), 2048 x 4096 (4.9 5.8 7.6 and 8.4 8.8
// 10.4, 8 are taken) and 1500 x 700 (4.0 4.8 6.7 and 7.3 7.8 9.6, 8 are taken), more at 8192 x 8192 (16.9 15.5 16.7 and 24.7 22.7 23.8, 4 are taken).
int few_waves(int features, int pitch)
{
    const int blocks = (features + 15) / 16;
    return blocks >= 512 || pitch < 8 * Q_STEP ? 4 : (blocks >= 256 || pitch < 16 * Q_STEP ? 8 : 16);
}
// Where a workgroup brings the tokens to 8 bits itself: two slices a thread at most, four for up to four tokens.  us, weights and tokens
// not in a cache, fused / in two launches: one token 2048 x 8192 6.4 / 8.8, 4096 x 2048 7.4 / 9.7, 1500 x 700 5.8 / 7.3; four 8.1 / 9.3,
// 9.0 / 10.2, 6.1 / 7.6; eight of 1024 x 1024 (two slices) 5.3 / 7.4, of 4096 x 2048 (four) 11.3 / 10.8, six of 1500 x 700 (three) 9.1 / 7.6.
bool few_fused(int tokens, int dim, int pitch, int waves)
{
    return tokens <= 16 && dim >= 8 && tokens * few_slices(pitch) <= (tokens <= 4 ? FEW_SLICES : 2) * waves * WAVE;
}
template <typename T>
void qfew_launch(const QFewArgs& a, bool fused, hipStream_t st)
{
    const dim3 grid((unsigned)((a.features + 15) / 16));
    auto with_waves = [&](auto w) {
        constexpr int W = decltype(w)::value;
        if (fused && a.tokens * few_slices(a.pitch) <= W * WAVE) hipLaunchKernelGGL((qfew_kernel<T, 1, W, 1>), grid, dim3(W * WAVE), 0, st, a);
        else if (fused && a.tokens * few_slices(a.pitch) <= 2 * W * WAVE) hipLaunchKernelGGL((qfew_kernel<T, 1, W, 2>), grid, dim3(W * WAVE), 0, st, a);
        else if (fused) hipLaunchKernelGGL((qfew_kernel<T, 1, W, FEW_SLICES>), grid, dim3(W * WAVE), 0, st, a);
        else if (a.tokens <= 16) hipLaunchKernelGGL((qfew_kernel<T, 1, W, 0>), grid, dim3(W * WAVE), 0, st, a);
        else hipLaunchKernelGGL((qfew_kernel<T, 2, W, 0>), grid, dim3(W * WAVE), 0, st, a);
    };
    const int w = few_waves(a.features, a.pitch);
    if (w == 4) with_waves(std::integral_constant<int, 4>{});
    else if (w == 8) with_waves(std::integral_constant<int, 8>{});
    else with_waves(std::integral_constant<int, 16>{});
}

// Tiles of 256, 128 or 64 by what a launch is modelled to take, in us: a start and an end, and steps that take as long as one
// workgroup alone needs for each of its rounds (1, 2 and 2 workgroups share a compute unit), or as the chip needs for all of
// them where that is more.  Fitted to 33 .. 16384 tokens at 2048 x 8192, 4096 x 2048, 768 x 3008 and 5120 x 2560 (dim x features).  us with 256 /
// 128 / 64: 256 tokens at 2048 x 8192 27.1 / 15.5 / 10.7, 512 28.2 / 17.1 / 19.7, 1024 31.5 / 24.1 / 36.8, 4096 76.2 / 89.1 / 137.5;
// 1024 at 4096 x 2048 49.6 / 25.5 / 17.4, 2048 52.0 / 28.7 / 33.4, 8192 69.6 / 80.5 / 122.0.
// Few tiles are bound by the latency of their requests and look three steps ahead: with weights and tokens not in a cache, the
// quantiser's launch included, 128 tokens at 4096 x 2048 16.2 us against 29.3 one step ahead (tiles of 64), 512 at 2048 x 8192 20.1
// against 25.4 (tiles of 128, of which two of one step ahead share a unit: 1024 tokens 34.5 against 29.6).
template <typename T>
void qgemm_launch(const QGemmArgs& a, hipStream_t st)
{
    auto tiles = [&](int t) { return (int64_t)((a.M + t - 1) / t) * ((a.N + t - 1) / t) * a.batch; };
    auto us = [&](int64_t n, int at_once, double ends, double alone, double each) {
        const double rounds = alone * (double)((n + at_once - 1) / at_once), all = each * (double)n;
        return ends + a.K / Q_STEP * (rounds > all ? rounds : all);
    };
    // tiles of 256 stay, so they take no more workgroups than units; of the others a launch may have no threads for as many
    const double never = 1e300, t256 = us(tiles(256), 256, 10.0, 1.13, 0.0082);
    const double t128 = tiles(128) * 256 > MOST_THREADS ? never : us(tiles(128), 512, 6.0, 0.56, 0.0023);
    const double t64 = tiles(64) * 256 > MOST_THREADS ? never : us(tiles(64), 512, 4.2, 0.27, 0.00095);
    if (t256 <= t128 && t256 <= t64)
        hipLaunchKernelGGL((qgemm_kernel<T, 4, 2, 2, 4, 2, true>), dim3((unsigned)(tiles(256) < 256 ? tiles(256) : 256)), dim3(512), 0, st, a);
    else if (t128 <= t64 && tiles(128) > 256) hipLaunchKernelGGL((qgemm_kernel<T, 2, 2, 2, 2, 2, false>), dim3((unsigned)tiles(128)), dim3(256), 0, st, a);
    else if (t128 <= t64) hipLaunchKernelGGL((qgemm_kernel<T, 2, 2, 2, 2, 4, false>), dim3((unsigned)tiles(128)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((qgemm_kernel<T, 2, 2, 1, 1, 4, false>), dim3((unsigned)tiles(64)), dim3(256), 0, st, a);
}

// ---- launches of the quantiser ------------------------------------------------------------------------
struct QuantSizes {
    int batch, L, dim, pitch;
    int chunks;   // of channels, sequence last
};

// One pass over tokens with the sequence last, where that is faster.  us, not in a cache, one pass / two: bf16, 70, 1000, 4100 and 16384 tokens of
// 2048 channels 4.7 7.0 9.8 34.2 / 9.7 13.7 17.3 33.3, of 4096 9.5 9.8 21.1 58.4 / 10.2 15.1 27.5 71.3; 1000 of 5120 11.8 / 16.6; float32 of
// 2048 8.7 8.8 15.4 38.4 / 9.2 13.8 23.7 55.2, of 4096 11.6 11.4 27.7 89.7 / 9.5 15.9 35.2 114; but 4100 of 5120 31.4 / 31.7 (float32 45.4 / 41.3) and
// 70 of 8192 15.7 / 10.8.  Wide tiles read longer pieces of rows, and take many tokens to fill the chip: tiles of 8 (or 16) and of 32 tokens (float32: 16 of
// 4096), bf16 4096 channels 1000 tokens 9.8 / 14.1, 6000 28.2 / 21.3, float32 2048 1000 8.8 / 10.2, 8192 28.9 / 20.3.
template <typename T>
bool quant_held(const QuantSizes& z, const T* x, int8_t* q, float* scale, hipStream_t st)
{
    constexpr bool NARROW = sizeof(T) == 2;
    const int tokens = z.batch * z.L;
    auto go = [&](auto threads, auto wide, auto r) {
        constexpr int THREADS = decltype(threads)::value, WIDE = decltype(wide)::value, R = decltype(r)::value;
        if (z.pitch > 4 * (THREADS / WIDE) * R) return false;
        const int tiles = (z.L + 8 * WIDE - 1) / (8 * WIDE);
        if ((int64_t)tiles * z.batch * THREADS > MOST_THREADS) return false;
        hipLaunchKernelGGL((quant_held_kernel<T, THREADS, WIDE, R>), dim3((unsigned)(tiles * z.batch)), dim3(THREADS), 0, st, x, q, scale, z.batch, z.dim, z.L,
                           z.pitch, tiles);
        return true;
    };
    typedef std::integral_constant<int, 1> one;
    typedef std::integral_constant<int, 2> two;
    typedef std::integral_constant<int, 4> four;
    constexpr std::integral_constant<int, 1024> most{};
    if constexpr (!NARROW)
        if (z.pitch > 1024 && z.pitch <= 2048 && tokens >= 6000) return go(most, four{}, two{});
    if (z.pitch <= 2048) return go(std::integral_constant<int, 256>{}, two{}, one{}) || go(std::integral_constant<int, 512>{}, two{}, one{}) || go(most, two{}, one{});
    if constexpr (NARROW) {
        if (z.pitch > 4096) return z.pitch <= 6144 && tokens <= 3000 && go(most, one{}, two{});
        if (tokens >= 4000) return go(most, four{}, four{});
    } else if (tokens >= 3000) {
        return go(most, two{}, two{});
    }
    return go(std::integral_constant<int, 512>{}, one{}, two{});
}
template <typename T>
void quant_launch(const QuantSizes& z, bool seq_last, const void* xv, int8_t* q, float* scale, uint32_t* tops, hipStream_t st)
{
    const T* x = static_cast<const T*>(xv);
    if (seq_last) {
        if (quant_held<T>(z, x, q, scale, st)) return;
        hipLaunchKernelGGL(quant_tops_kernel<T>, dim3((unsigned)((z.L + 255) / 256), (unsigned)z.chunks, (unsigned)z.batch), dim3(256), 0, st, x, tops, z.batch,
                           z.dim, z.L);
        hipLaunchKernelGGL(quant_turn_kernel<T>, dim3((unsigned)((z.L + TURN_TOKENS - 1) / TURN_TOKENS), (unsigned)(z.pitch / Q_STEP), (unsigned)z.batch), dim3(256), 0, st, x, tops,
                           q, scale, z.batch, z.dim, z.L, z.pitch, z.chunks);
        return;
    }
    const int rows = z.batch * z.L;
    // f(first row, rows) for as many rows at a time as a launch has threads for
    auto in_parts = [&](int lanes, auto f) {
        const int most = (int)(MOST_THREADS / lanes / 4 * 4);
        for (int r = 0; r < rows; r += min(most, rows - r)) f(r, min(most, rows - r));
    };
    auto go = [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, V = decltype(v)::value, SIDE = (G > 256 ? G : 256) / G;
        in_parts(G, [&](int r, int n) {
            hipLaunchKernelGGL((quant_rows_kernel<T, G, V>), dim3((unsigned)((n + SIDE - 1) / SIDE)), dim3(G > 256 ? G : 256), 0, st, x + (int64_t)r * z.dim,
                               q + (int64_t)r * z.pitch, scale + r, n, z.dim, z.pitch);
        });
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
    else in_parts(1024, [&](int r, int n) {
        hipLaunchKernelGGL(quant_rows_wide_kernel<T>, dim3((unsigned)n), dim3(1024), 0, st, x + (int64_t)r * z.dim, q + (int64_t)r * z.pitch, scale + r, z.dim, z.pitch);
    });
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
    bool x_last = p->flags & SS_Q_X_SEQ_LAST, out_last = p->flags & SS_Q_OUT_SEQ_LAST;
    const bool done = p->flags & SS_Q_X_QUANTISED, hb = p->flags & SS_Q_HAS_BIAS;
    if (x_last && done) return SS_ERR_UNSUPPORTED;
    if (p->batch == 0 || p->seqlen == 0) return SS_OK;
    if ((x_last || out_last) && p->batch > 65535) return SS_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)p->batch * p->seqlen;
    // what the product's tiles, of at least 64 x 64, are numbered with
    const int64_t tm = ((out_last ? p->features : rows) + 63) / 64, tn = ((out_last ? p->seqlen : p->features) + 63) / 64;
    if (tm * tn > 0x7fffffff / (out_last ? p->batch : 1)) return SS_ERR_UNSUPPORTED;
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
    if (p->seqlen == 1) x_last = out_last = false;   // the two orders are one
    const int pitch = (int)ss_quant_pitch(p->dim);
    const int8_t* q = static_cast<const int8_t*>(p->x);
    const float* q_scale = p->x_scale;
    // (16 features and 256 threads a workgroup where there are as many features as that)
    const bool few = rows <= ss::FEW_TOKENS && !out_last && p->features <= ss::MOST_THREADS / 16;
    const bool fused = few && !done && !x_last && ss::few_fused((int)rows, p->dim, pitch, ss::few_waves(p->features, pitch));
    if (!done && !fused) {
        const ss::QuantSizes z = {p->batch, p->seqlen, p->dim, pitch, chunks_of(p->dim)};
        quantise(z, x_last, p->io_dtype, p->x, reinterpret_cast<int8_t*>(ws + s.q), reinterpret_cast<float*>(ws + s.scale), ws + s.tops, st);
        q = reinterpret_cast<const int8_t*>(ws + s.q);
        q_scale = reinterpret_cast<const float*>(ws + s.scale);
    }
    if (few) {
        const ss::QFewArgs f = {(int)rows, p->features, p->dim, pitch, p->x, q, q_scale, static_cast<const int8_t*>(p->weight), p->scale, hb ? p->bias : nullptr, p->out};
        if (p->io_dtype == SS_BF16) ss::qfew_launch<ss::bf16_t>(f, fused, st);
        else ss::qfew_launch<float>(f, fused, st);
        return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
    }
    ss::QGemmArgs g{};
    g.K = pitch;
    g.bias = hb ? p->bias : nullptr;
    g.C = p->out;
    const int8_t* w = static_cast<const int8_t*>(p->weight);
    g.batch = 1;
    if (out_last) {
        g.M = p->features; g.N = p->seqlen;
        g.A = w; g.a_scale = p->scale;
        g.B = q; g.b_scale = q_scale;
        g.b_batch = (int64_t)p->seqlen * pitch;
        g.bs_batch = p->seqlen;
        g.c_batch = (int64_t)p->features * p->seqlen;
        g.bias_m = 1;
        g.batch = p->batch;
    } else {
        g.M = (int)rows; g.N = p->features;
        g.A = q; g.a_scale = q_scale;
        g.B = w; g.b_scale = p->scale;
    }
    if (p->io_dtype == SS_BF16) ss::qgemm_launch<ss::bf16_t>(g, st);
    else ss::qgemm_launch<float>(g, st);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
