// Embedding of token ids and its gradient for gfx950, with the C-ABI entry points (see include/ss_embed.h).
//
// Forward: rows of a table are copied, so it is bound by HBM (and for few tokens by a launch).
// Backward: every row of the table's gradient is written, most of them with zeros, and every token's row is read once.  To add up a row
// without atomics, and always in the same order, the tokens are sorted by id first: a radix sort, least digit first and stable, so
// that the tokens of an id stay in order.  Its launches are short and leave most of the chip idle, so each also fills a share
// of the gradient with zeros.  Sorted tokens are then cut into pieces of equal length, whatever their ids (one id may have all tokens), a
// group of lanes adds a piece up, writes the rows that lie within it, and leaves the sums of the ids that it shares with its
// neighbours to a second kernel, which adds those of an id in order.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ss_embed.h"
#include "ss_slices.h"

namespace ss {

struct EmbedArgs {
    int tokens, vocab, dim;
    float scale;
    const void *ids, *table, *dout;
    void *out, *dtable;
    // sorting
    const int *key_in, *pos_in;   // null: the ids themselves, in order
    int *key_out, *pos_out;
    int* hist;                    // (tiles, 2^digit)
    int tile, tiles;              // tokens of a tile, their number
    int shift, digit;             // bits below the digit, bits of it
    int64_t fill_from, fill_to;   // elements of dtable that the launch sets to zero
    // sums
    const int *key, *pos;
    int piece, pieces;            // sorted tokens of a piece, their number
    float* part;                  // (pieces, 2, dim): of an id that began before the piece, and of one that goes on behind it
};

// ---- forward --------------------------------------------------------------------------------------
template <typename I>
__device__ __forceinline__ int id_of(const void* ids, int t, int vocab)   // vocab for what is outside
{
    const I v = static_cast<const I*>(ids)[t];
    return v >= 0 && v < vocab ? (int)v : vocab;
}
// slices of rows that are read one by one: the last is read from further ahead and shifted into place
template <typename T>
__device__ __forceinline__ void row_slice(const T* row, int at, int dim, float (&v)[8])
{
    const bool whole = dim % 8 == 0;
    const int limit = slice_limit(dim, whole);
    typename io8<T>::raw r = slice_request<T, true>(row, at, dim, limit);
    slice_settle<T>(r, at, dim, limit, whole);
    io8<T>::unpack(r, v);
}

// G lanes a token, a slice of eight a lane and step.
template <typename E, typename T, typename I, int G>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedArgs a)
{
    constexpr int SIDE = 256 / G;
    const int gl = threadIdx.x % G, D = a.dim;
    for (int64_t t = (int64_t)blockIdx.x * SIDE + threadIdx.x / G; t < a.tokens; t += (int64_t)gridDim.x * SIDE) {
        const int id = id_of<I>(a.ids, (int)t, a.vocab);
        const E* row = static_cast<const E*>(a.table) + (int64_t)id * D;
        T* out = static_cast<T*>(a.out) + t * D;
        for (int at = gl * 8; at < D; at += G * 8) {
            float v[8] = {};
            if (id < a.vocab) row_slice<E>(row, at, D, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= a.scale;
            slice_store<T>(out, at, D - at, v);
        }
    }
}

// ---- sorting --------------------------------------------------------------------------------------
constexpr int SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / WAVE;
constexpr int DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;
constexpr int FILL_WORKGROUPS = 2048;

// The workgroups behind the sorting ones set a share of the gradient to zero.
template <typename E>
__device__ __forceinline__ void fill(const EmbedArgs& a, int64_t wg, int64_t wgs)
{
    E* const to = static_cast<E*>(a.dtable);
    constexpr int N = 16 / sizeof(E);
    for (int64_t k = a.fill_from + (wg * SORT_THREADS + threadIdx.x) * N; k < a.fill_to; k += wgs * SORT_THREADS * N) {
        if (k + N <= a.fill_to) {
            store_any(to + k, 0u, u32x4{0u, 0u, 0u, 0u});
        } else {
            for (int j = 0; k + j < a.fill_to; ++j) to[k + j] = (E)0;
        }
    }
}
template <typename I>
__device__ __forceinline__ int sort_key(const EmbedArgs& a, int t)
{
    return a.key_in ? a.key_in[t] : id_of<I>(a.ids, t, a.vocab);
}

// How many tokens of each tile have each digit.
template <typename E, typename I>
__global__ __launch_bounds__(SORT_THREADS) void embed_count_kernel(EmbedArgs a)
{
    if ((int)blockIdx.x >= a.tiles) return fill<E>(a, (int64_t)blockIdx.x - a.tiles, (int64_t)gridDim.x - a.tiles);
    __shared__ int count[DIGITS];
    const int digits = 1 << a.digit;
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) count[d] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * a.tile;
    const int to = (int)min(from + a.tile, (int64_t)a.tokens);
    for (int t = (int)from + threadIdx.x; t < to; t += SORT_THREADS) atomicAdd(&count[(sort_key<I>(a, t) >> a.shift) & (digits - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) a.hist[blockIdx.x * digits + d] = count[d];
}

// Every token to its place: behind all tokens with lower digits, those of earlier tiles, of earlier waves (each has a stretch of the tile) and of
// earlier lanes with the same.  64 tokens a wave and step; those of a wave with the same digit are found by ballots of its bits.
template <typename E, typename I>
__global__ __launch_bounds__(SORT_THREADS) void embed_place_kernel(EmbedArgs a)
{
    if ((int)blockIdx.x >= a.tiles) return fill<E>(a, (int64_t)blockIdx.x - a.tiles, (int64_t)gridDim.x - a.tiles);
    __shared__ int place[SORT_WAVES][DIGITS];   // counts, then the next free place of each wave's
    __shared__ int sums[SORT_WAVES];
    const int digits = 1 << a.digit, wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    for (int d = threadIdx.x; d < SORT_WAVES * DIGITS; d += SORT_THREADS) (&place[0][0])[d] = 0;
    __syncthreads();
    const int stretch = a.tile / SORT_WAVES;
    const int64_t from = (int64_t)blockIdx.x * a.tile + wave * stretch;
    const int to = (int)min(from + stretch, (int64_t)a.tokens);
    for (int64_t t = from + lane; t < to; t += WAVE) atomicAdd(&place[wave][(sort_key<I>(a, (int)t) >> a.shift) & (digits - 1)], 1);
    // tokens with the digits of a thread, two beside each other: all of them, and those of earlier tiles
    int all[2] = {0, 0}, before[2] = {0, 0};
    const int d0 = threadIdx.x * 2;
    if (d0 < digits) {
        for (int k = 0; k < a.tiles; ++k) {
            const int2 c = *reinterpret_cast<const int2*>(a.hist + k * digits + d0);
            all[0] += c.x;
            all[1] += c.y;
            if (k < (int)blockIdx.x) {
                before[0] += c.x;
                before[1] += c.y;
            }
        }
    }
    int up = all[0] + all[1];   // of this thread's digits and those before, within the wave
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) {
        const int v = __shfl_up(up, s);
        if (lane >= s) up += v;
    }
    if (lane == WAVE - 1) sums[wave] = up;
    __syncthreads();
    int base = up - all[0] - all[1];
    for (int w = 0; w < wave; ++w) base += sums[w];
    if (d0 < digits) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            int at = base + before[j];
            base += all[j];
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int n = place[w][d0 + j];
                place[w][d0 + j] = at;
                at += n;
            }
        }
    }
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += WAVE) {
        const int64_t t = t0 + lane;
        const bool valid = t < to;
        const int key = valid ? sort_key<I>(a, (int)t) : 0;
        const int d = (key >> a.shift) & (digits - 1);
        uint64_t same = __ballot(valid);
        for (int b = 0; b < a.digit; ++b) {
            const bool on = (d >> b) & 1;
            const uint64_t bal = __ballot(on);
            same &= on ? bal : ~bal;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int to_place = place[wave][d] + rank;
        __builtin_amdgcn_wave_barrier();   // all lanes have read before the last of each digit writes
        if (valid) {
            if ((same >> lane) == 1ull) place[wave][d] = to_place + 1;
            a.key_out[to_place] = key;
            a.pos_out[to_place] = a.pos_in ? a.pos_in[t] : (int)t;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- sums -----------------------------------------------------------------------------------------
template <typename E>
__device__ __forceinline__ void store_row(const EmbedArgs& a, int id, int at, const float (&v)[8])
{
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = v[j] * a.scale;
    slice_store<E>(static_cast<E*>(a.dtable) + (int64_t)id * a.dim, at, a.dim - at, o);
}
__device__ __forceinline__ float* part_of(const EmbedArgs& a, int64_t piece, int which) { return a.part + (piece * 2 + which) * a.dim; }

template <typename E, typename T, int G>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a)
{
    constexpr int SIDE = 256 / G, AHEAD = 8;
    const int64_t piece = (int64_t)blockIdx.x * SIDE + threadIdx.x / G;
    const int at = (blockIdx.y * G + threadIdx.x % G) * 8;
    if (piece >= a.pieces || at >= a.dim) return;
    const int i0 = (int)(piece * a.piece), i1 = (int)min((int64_t)i0 + a.piece, (int64_t)a.tokens);
    int id = a.key[i0];
    if (id >= a.vocab) return;   // ids outside the table come last
    bool began = i0 == 0 || a.key[i0 - 1] != id;
    float acc[8] = {};
    auto finish = [&](bool goes_on) {
        if (id >= a.vocab) return;
        if (began && !goes_on) store_row<E>(a, id, at, acc);
        else slice_store<float>(part_of(a, piece, began ? 1 : 0), at, a.dim - at, acc);
    };
    const bool whole = a.dim % 8 == 0;
    const int limit = slice_limit(a.dim, whole);
    for (int i = i0; i < i1; i += AHEAD) {
        typename io8<T>::raw r[AHEAD];
        int key[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = min(i + j, i1 - 1);
            key[j] = a.key[k];
            r[j] = slice_request<T, true>(static_cast<const T*>(a.dout) + (int64_t)a.pos[k] * a.dim, at, a.dim, limit);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (i + j >= i1) break;
            if (key[j] != id) {
                finish(false);
                id = key[j];
                began = true;
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = 0.0f;
            }
            float v[8];
            slice_settle<T>(r[j], at, a.dim, limit, whole);
            io8<T>::unpack(r[j], v);
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] += v[c];
        }
    }
    finish(i1 < a.tokens && a.key[i1] == id);
}

// The rows of ids that several pieces share, by the piece that they begin in.
template <typename E, int G>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a)
{
    constexpr int SIDE = 256 / G;
    const int64_t piece = (int64_t)blockIdx.x * SIDE + threadIdx.x / G;
    const int at = (blockIdx.y * G + threadIdx.x % G) * 8;
    if (piece >= a.pieces - 1 || at >= a.dim) return;
    const int i0 = (int)(piece * a.piece), i1 = i0 + a.piece;
    const int id = a.key[i1 - 1];
    if (id >= a.vocab || a.key[i1] != id || (i0 > 0 && a.key[i0 - 1] == id)) return;
    int low = i1, high = a.tokens;   // the id's tokens end in (low, high]
    while (high - low > 1) {
        const int mid = low + (high - low) / 2;
        if (a.key[mid] == id) low = mid;
        else high = mid;
    }
    const int64_t last = low / a.piece;
    float acc[8], v[8];
    row_slice<float>(part_of(a, piece, 1), at, a.dim, acc);
#pragma unroll 8
    for (int64_t k = piece + 1; k <= last; ++k) {
        row_slice<float>(part_of(a, k, 0), at, a.dim, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
    }
    store_row<E>(a, id, at, acc);
}

// ---- sizes ----------------------------------------------------------------------------------------
template <typename F>
void with_lanes(int dim, F go)   // lanes of a row: as many as it has slices, up to a workgroup
{
    const int n = (dim + 7) / 8;
    if (n <= 8) go(std::integral_constant<int, 8>{});
    else if (n <= 64) go(std::integral_constant<int, 64>{});
    else go(std::integral_constant<int, 256>{});
}
struct EmbedPlan {
    int passes, digit, tile, tiles, piece, pieces;
    size_t key[2], pos[2], hist, part, total;   // offsets in bytes
};
EmbedPlan embed_plan(int tokens, int vocab, int dim)
{
    EmbedPlan p{};
    int bits = 1;
    while (((int64_t)vocab >> bits) != 0) ++bits;   // of ids up to vocab, which stands for those outside
    p.passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
    p.digit = (bits + p.passes - 1) / p.passes;
    // tiles of 1024 tokens, of more where there would be over 64 (every tile reads all tiles' counts)
    const int64_t tile = std::max((int64_t)1024, ((int64_t)tokens + 63) / 64);
    p.tile = (int)((tile + SORT_THREADS - 1) / SORT_THREADS * SORT_THREADS);
    p.tiles = (int)(((int64_t)tokens + p.tile - 1) / p.tile);
    // pieces of 32 tokens, of more where there would be over 4096 (an id may have all of them)
    p.piece = 32;
    while (((int64_t)tokens + p.piece - 1) / p.piece > 4096) p.piece *= 2;
    p.pieces = (int)(((int64_t)tokens + p.piece - 1) / p.piece);
    auto take = [&](size_t bytes) {
        const size_t at = p.total;
        p.total += (bytes + 255) / 256 * 256;
        return at;
    };
    for (int k = 0; k < 2; ++k) {
        p.key[k] = take((size_t)tokens * 4);
        p.pos[k] = take((size_t)tokens * 4);
    }
    p.hist = take((size_t)p.tiles * DIGITS * 4);
    p.part = take((size_t)p.pieces * 2 * dim * 4);
    return p;
}

template <typename E, typename T, typename I>
void embed_forward(const EmbedArgs& a, hipStream_t st)
{
    with_lanes(a.dim, [&](auto g) {
        constexpr int G = decltype(g)::value, SIDE = 256 / G;
        const int64_t n = ((int64_t)a.tokens + SIDE - 1) / SIDE;
        hipLaunchKernelGGL((embed_fwd_kernel<E, T, I, G>), dim3((unsigned)std::min(n, (int64_t)8192)), dim3(256), 0, st, a);
    });
}
template <typename E, typename T, typename I>
void embed_backward(EmbedArgs a, char* ws, hipStream_t st)
{
    const EmbedPlan p = embed_plan(a.tokens, a.vocab, a.dim);
    const int64_t all = (int64_t)a.vocab * a.dim;
    const int shares = a.tokens ? 2 * p.passes : 1;
    a.hist = reinterpret_cast<int*>(ws + p.hist);
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.tile = p.tile; a.tiles = p.tiles; a.digit = p.digit;
    a.piece = p.piece; a.pieces = p.pieces;
    for (int k = 0; k < shares; ++k) {
        // shares of whole 16-byte words from the start
        a.fill_from = all / shares * k / 8 * 8;
        a.fill_to = k == shares - 1 ? all : all / shares * (k + 1) / 8 * 8;
        const int64_t words = (a.fill_to - a.fill_from) * (int64_t)sizeof(E) / (16 * SORT_THREADS * 4) + 1;
        const dim3 grid((unsigned)(p.tiles + std::min(words, (int64_t)FILL_WORKGROUPS)));
        const int pass = k / 2, to = pass % 2;
        a.shift = pass * p.digit;
        a.key_in = pass ? reinterpret_cast<int*>(ws + p.key[1 - to]) : nullptr;
        a.pos_in = pass ? reinterpret_cast<int*>(ws + p.pos[1 - to]) : nullptr;
        a.key_out = reinterpret_cast<int*>(ws + p.key[to]);
        a.pos_out = reinterpret_cast<int*>(ws + p.pos[to]);
        if (k % 2 == 0) hipLaunchKernelGGL((embed_count_kernel<E, I>), grid, dim3(SORT_THREADS), 0, st, a);
        else hipLaunchKernelGGL((embed_place_kernel<E, I>), grid, dim3(SORT_THREADS), 0, st, a);
    }
    if (!a.tokens) return;
    a.key = a.key_out;
    a.pos = a.pos_out;
    with_lanes(a.dim, [&](auto g) {
        constexpr int G = decltype(g)::value, SIDE = 256 / G;
        const dim3 grid((unsigned)((p.pieces + SIDE - 1) / SIDE), (unsigned)((a.dim + G * 8 - 1) / (G * 8)));
        hipLaunchKernelGGL((embed_sum_kernel<E, T, G>), grid, dim3(256), 0, st, a);
        if (p.pieces > 1) hipLaunchKernelGGL((embed_join_kernel<E, G>), grid, dim3(256), 0, st, a);
    });
}
template <typename F>
void with_types(const ss_embed_params* p, F go)
{
    auto ids = [&](auto e, auto t) {
        if (p->flags & SS_EMBED_IDS_32) go(e, t, (int32_t)0);
        else go(e, t, (int64_t)0);
    };
    auto io = [&](auto e) {
        if (p->io_dtype == SS_F32) ids(e, float());
        else ids(e, bf16_t());
    };
    if (p->table_dtype == SS_F32) io(float());
    else io(bf16_t());
}

}  // namespace ss

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t bytes_of(int32_t dtype) { return dtype == SS_BF16 ? 2 : 4; }
constexpr int32_t EMBED_MOST = 0x7fffffff - 65536;      // room for the last steps of the kernels' loops
constexpr int32_t EMBED_WIDEST = 65535 * 2048;          // columns that the workgroups along y of a launch reach

int check_embed(const ss_embed_params* p)
{
    if (!p) return SS_ERR_NULL;
    if (p->tokens < 0 || p->vocab < 1 || p->dim < 1) return SS_ERR_SHAPE;
    if ((p->table_dtype != SS_F32 && p->table_dtype != SS_BF16) || (p->io_dtype != SS_F32 && p->io_dtype != SS_BF16)) return SS_ERR_UNSUPPORTED;
    if ((p->flags & ~(uint32_t)SS_EMBED_IDS_32) || !std::isfinite(p->scale)) return SS_ERR_UNSUPPORTED;
    if (p->tokens > EMBED_MOST || p->vocab > EMBED_MOST || p->dim > EMBED_WIDEST) return SS_ERR_UNSUPPORTED;
    if (p->tokens > 0 && !p->ids) return SS_ERR_NULL;
    if (!aligned_to(p->ids, p->flags & SS_EMBED_IDS_32 ? 4 : 8)) return SS_ERR_ALIGN;
    return SS_OK;
}
ss::EmbedArgs embed_args(const ss_embed_params* p)
{
    ss::EmbedArgs a{};
    a.tokens = p->tokens; a.vocab = p->vocab; a.dim = p->dim; a.scale = p->scale; a.ids = p->ids;
    return a;
}

}  // namespace

extern "C" {

int ss_embed_fwd(const ss_embed_params* p, void* stream)
{
    const int rc = check_embed(p);
    if (rc != SS_OK) return rc;
    if (p->tokens == 0) return SS_OK;
    if (!p->table || !p->out) return SS_ERR_NULL;
    if (!aligned_to(p->table, bytes_of(p->table_dtype)) || !aligned_to(p->out, bytes_of(p->io_dtype))) return SS_ERR_ALIGN;
    ss::EmbedArgs a = embed_args(p);
    a.table = p->table;
    a.out = p->out;
    ss::with_types(p, [&](auto e, auto t, auto i) {
        ss::embed_forward<decltype(e), decltype(t), decltype(i)>(a, static_cast<hipStream_t>(stream));
    });
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

size_t ss_embed_workspace_bytes(const ss_embed_params* p)
{
    if (!p || p->tokens < 1 || p->vocab < 1 || p->dim < 1) return 0;
    return ss::embed_plan(p->tokens, p->vocab, p->dim).total;
}

int ss_embed_bwd(const ss_embed_bwd_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    const ss_embed_params* f = &p->fwd;
    const int rc = check_embed(f);
    if (rc != SS_OK) return rc;
    if (!p->dtable || (f->tokens > 0 && !p->dout)) return SS_ERR_NULL;
    if (!aligned_to(p->dtable, bytes_of(f->table_dtype)) || !aligned_to(p->dout, bytes_of(f->io_dtype))) return SS_ERR_ALIGN;
    if (f->tokens > 0) {
        if (!p->workspace || p->workspace_bytes < ss_embed_workspace_bytes(f)) return SS_ERR_WORKSPACE;
        if (!aligned_to(p->workspace, 256)) return SS_ERR_ALIGN;
    }
    ss::EmbedArgs a = embed_args(f);
    a.dout = p->dout;
    a.dtable = p->dtable;
    ss::with_types(f, [&](auto e, auto t, auto i) {
        ss::embed_backward<decltype(e), decltype(t), decltype(i)>(a, static_cast<char*>(p->workspace), static_cast<hipStream_t>(stream));
    });
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
