// Embedding of token ids and its gradient for gfx950, with the C-ABI entry points (see include/ss_embed.h).
//
// Forward: rows of a table are copied, so it is bound by HBM (16384 rows of 2048 float32 as bf16, 201 MB, 31 us, 6.4 TB/s, of ids that
// are drawn evenly; as in text, where every other row has been read before, 24) and for few tokens by a launch.
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
    int* shared;                  // their number, and the pieces that ids begin in which several share
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
    const bool whole = D % 8 == 0;
    const int limit = slice_limit(D, whole);
    int64_t t = (int64_t)blockIdx.x * SIDE;
    t += G >= WAVE ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
    for (; t < a.tokens; t += (int64_t)gridDim.x * SIDE) {
        const int id = id_of<I>(a.ids, (int)t, a.vocab);
        const bool there = id < a.vocab;
        const E* row = static_cast<const E*>(a.table) + (int64_t)(there ? id : 0) * D;
        T* out = static_cast<T*>(a.out) + t * D;
        for (int at = gl * 8; at < D; at += G * 8) {
            float f[8];
            row_slice<E>(row, at, D, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = there ? f[j] * a.scale : 0.0f;
            slice_store<T>(out, at, D - at, f);
        }
    }
}

// ---- sorting --------------------------------------------------------------------------------------
constexpr int SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / WAVE;
constexpr int DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;
constexpr int FILL_STORES = 4;                 // of 16 bytes, of a thread
constexpr int64_t FILL_WORKGROUPS = 1 << 20;

// The workgroups behind the sorting ones set a share of the gradient to zero, in stretches of four words a thread.  PAST: past the caches.
// 105 MB beside the sort of 16384 ids 18 us a launch, 5.7 TB/s; the same zeros in a launch of their own 15.
template <typename E, bool PAST>
__device__ __forceinline__ void fill(const EmbedArgs& a, int64_t wg, int64_t wgs)
{
    E* const to = static_cast<E*>(a.dtable);
    constexpr int N = 16 / sizeof(E), STRETCH = SORT_THREADS * N * FILL_STORES;
    for (int64_t k0 = a.fill_from + wg * STRETCH; k0 < a.fill_to; k0 += wgs * STRETCH) {
#pragma unroll
        for (int u = 0; u < FILL_STORES; ++u) {
            const int64_t k = k0 + (u * SORT_THREADS + threadIdx.x) * N;
            if (k + N <= a.fill_to) {
                if constexpr (PAST) store_past(to + k, u32x4{0u, 0u, 0u, 0u});
                else store_any(to + k, 0u, u32x4{0u, 0u, 0u, 0u});
            } else {
                for (int j = 0; k + j < a.fill_to; ++j) to[k + j] = (E)0;
            }
        }
    }
}
template <typename I>
__device__ __forceinline__ int sort_key(const EmbedArgs& a, int t)
{
    return a.key_in ? a.key_in[t] : id_of<I>(a.ids, t, a.vocab);
}

// How many tokens of each tile have each digit.
template <typename E, typename I, bool PAST>
__global__ __launch_bounds__(SORT_THREADS) void embed_count_kernel(EmbedArgs a)
{
    if ((int)blockIdx.x >= a.tiles) return fill<E, PAST>(a, (int64_t)blockIdx.x - a.tiles, (int64_t)gridDim.x - a.tiles);
    __shared__ int count[DIGITS];
    const int digits = 1 << a.digit;
    if (blockIdx.x == 0 && threadIdx.x == 0) a.shared[0] = 0;
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
template <typename E, typename I, bool PAST>
__global__ __launch_bounds__(SORT_THREADS) void embed_place_kernel(EmbedArgs a)
{
    if ((int)blockIdx.x >= a.tiles) return fill<E, PAST>(a, (int64_t)blockIdx.x - a.tiles, (int64_t)gridDim.x - a.tiles);
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
    if (a.tiles == 1) {   // no launch has counted
        if (threadIdx.x == 0) a.shared[0] = 0;
        __syncthreads();
        for (int w = 0; d0 < digits && w < SORT_WAVES; ++w) {
            all[0] += place[w][d0];
            all[1] += place[w][d0 + 1];
        }
    } else if (d0 < digits) {
        for (int k0 = 0; k0 < a.tiles; k0 += 8) {
            int2 c[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = *reinterpret_cast<const int2*>(a.hist + min(k0 + k, a.tiles - 1) * digits + d0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool real = k0 + k < a.tiles, early = k0 + k < (int)blockIdx.x;
                all[0] += real ? c[k].x : 0;
                all[1] += real ? c[k].y : 0;
                before[0] += early ? c[k].x : 0;
                before[1] += early ? c[k].y : 0;
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
    constexpr int AHEAD = 4;
    for (int64_t t0 = from; t0 < to; t0 += AHEAD * WAVE) {
        int keys[AHEAD], places[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int t = (int)min(t0 + u * WAVE + lane, (int64_t)to - 1);
            keys[u] = sort_key<I>(a, t);
            places[u] = a.pos_in ? a.pos_in[t] : t;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const bool valid = t0 + u * WAVE + lane < to;
            const int d = (keys[u] >> a.shift) & (digits - 1);
            uint64_t same = __ballot(valid);
            for (int b = 0; b < a.digit; ++b) {
                const bool on = (d >> b) & 1;
                const uint64_t bal = __ballot(on);
                same &= on ? bal : ~bal;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const int at = place[wave][d] + rank;
            wave_lds_fence();   // all lanes have read before the last of each digit writes
            if (valid) {
                if ((same >> lane) == 1ull) place[wave][d] = at + 1;
                a.key_out[at] = keys[u];
                a.pos_out[at] = places[u];
            }
            wave_lds_fence();
        }
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

// A wave has a piece and 512 columns.  It adds up every id whose tokens begin in the piece, and goes on behind its end where no more than SPILL tokens of the
// last one follow; of longer ones it leaves its share.  The share of an id that began before the piece: the same, and nothing where the wave
// before goes on to its end.  Ids and places come 64 at once, a lane each, eight rows are requested at once.  Bound by HBM: 65536 rows of 1024 bf16 (135 MB) for
// 256 ids 25 to 30 us, 4.5 TB/s and more; 16384 of 2048 for 51200 ids, most of which have one row or none (195 MB), 41, as in text 32.
constexpr int SPILL = 8;   // a piece has that many at least (1024 tokens of 1024 columns: 5.4 us, with 16 7.4)
template <typename E, typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a)
{
    constexpr int AHEAD = 8, BLOCK = 32;
    const int piece = __builtin_amdgcn_readfirstlane(blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const int at = (blockIdx.y * WAVE + lane) * 8;
    if (piece >= a.pieces) return;
    const int N = a.tokens, i0 = piece * a.piece, i1 = (int)min((int64_t)i0 + a.piece, (int64_t)N);
    auto key = [&](int64_t i) { return a.key[min(max(i, (int64_t)0), (int64_t)N - 1)]; };
    const int first = key(i0), before = key(i0 - 1), far_before = key((int64_t)i0 - a.piece - 1), spilt = key((int64_t)i0 + SPILL);
    const int last = key(i1 - 1), next = key(i1), far_next = key((int64_t)i1 + SPILL);
    const int around0 = key((int64_t)i0 + lane), around1 = key((int64_t)i1 + lane);   // from the piece's begin and end on
    if (first >= a.vocab) return;   // ids outside the table come last
    bool began = i0 == 0 || before != first;
    int from = i0, to = i1;
    if (!began && (i0 - a.piece - 1 < 0 || far_before != first) && ((int64_t)i0 + SPILL >= N || spilt != first)) {
        from += __ffsll((long long)~__ballot(around0 == first && i0 + lane < i1)) - 1;   // up to SPILL of them: the wave before adds them
        began = true;
        if (from >= i1) return;
    }
    bool goes_on = i1 < N && next == last;
    if (goes_on && (began || last != first) && ((int64_t)i1 + SPILL >= N || far_next != last)) {
        to += __ffsll((long long)~__ballot(around1 == last && (int64_t)i1 + lane < N)) - 1;
        goes_on = false;
    }
    const bool whole = a.dim % 8 == 0, some = at < a.dim;
    const int limit = slice_limit(a.dim, whole);
    float acc[8] = {};
    int id = -1;
    auto finish = [&](bool open) {
        if (id < 0 || id >= a.vocab || !some) return;
        if (began && !open) store_row<E>(a, id, at, acc);
        else slice_store<float>(part_of(a, piece, began ? 1 : 0), at, a.dim - at, acc);
    };
    for (int b = from; b < to; b += BLOCK) {
        const int keys = key(b + lane), places = a.pos[min(b + lane, N - 1)];
        for (int j0 = 0; j0 < BLOCK && b + j0 < to; j0 += AHEAD) {
            typename io8<T>::raw r[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int place = __builtin_amdgcn_readlane(places, min(j0 + j, to - 1 - b));
                r[j] = slice_request<T, true>(static_cast<const T*>(a.dout) + (int64_t)place * a.dim, at, a.dim, limit);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (b + j0 + j >= to) break;
                const int k = __builtin_amdgcn_readlane(keys, j0 + j);
                if (k != id) {
                    if (id >= 0) {
                        finish(false);
                        began = true;
                    }
                    id = k;
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
    }
    finish(goes_on);
    if (goes_on && began && id < a.vocab && blockIdx.y == 0 && lane == 0) a.shared[1 + atomicAdd(&a.shared[0], 1)] = piece;   // in any order: each is a row of its own
}

// The rows of ids that go on for more than SPILL tokens behind the piece that they begin in: a workgroup for 512 columns of one, whose waves
// take a share of its pieces each (four waves instead of 16: 38 us against 17 where one id has 336 pieces, as in text, 6 against 10 where all
// have 16).  Bound by the few workgroups' trips to memory: 4 us without any such id, 6 with some, 36 where one id has all of 65536 tokens.
constexpr int JOIN_WAVES = 16, JOIN_WORKGROUPS = 256;
template <typename E>
__global__ __launch_bounds__(JOIN_WAVES * WAVE) void embed_join_kernel(EmbedArgs a)
{
    __shared__ float sums[JOIN_WAVES][WAVE][9];
    const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, rows = a.shared[0];
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const int piece = a.shared[1 + row];
        const int id = a.key[(piece + 1) * a.piece - 1];
        // the last piece that begins with the id: 64 are looked at at once
        int last = piece + 1;
        for (;;) {
            const int k = last + 1 + lane;
            const uint64_t on = __ballot(k < a.pieces && a.key[(int64_t)min(k, a.pieces - 1) * a.piece] == id);
            if (on == ~0ull) {
                last += WAVE;
                continue;
            }
            last += __ffsll((long long)~on) - 1;
            break;
        }
        const int at = (blockIdx.y * WAVE + lane) * 8, parts = last - piece + 1;   // the first has its own place
        float acc[8] = {};
        if (at < a.dim) {
            const int from = (int)((int64_t)parts * wave / JOIN_WAVES), to = (int)((int64_t)parts * (wave + 1) / JOIN_WAVES);
            const bool whole = a.dim % 8 == 0;
            const int limit = slice_limit(a.dim, whole);
            for (int k0 = from; k0 < to; k0 += 8) {
                typename io8<float>::raw r[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = min(k0 + j, to - 1);
                    r[j] = slice_request<float, true>(part_of(a, piece + k, k == 0 ? 1 : 0), at, a.dim, limit);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (k0 + j >= to) break;
                    float v[8];
                    slice_settle<float>(r[j], at, a.dim, limit, whole);
                    io8<float>::unpack(r[j], v);
#pragma unroll
                    for (int c = 0; c < 8; ++c) acc[c] += v[c];
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) sums[wave][lane][c] = acc[c];
        // halves of the waves' sums onto halves, each a fixed pair
        for (int half = JOIN_WAVES / 2; half > 0; half /= 2) {
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int c = 0; c < 8; ++c) sums[wave][lane][c] = acc[c] += sums[wave + half][lane][c];
            }
        }
        if (wave == 0 && at < a.dim) store_row<E>(a, id, at, acc);
        __syncthreads();   // the next row's sums come into the same place
    }
}

// ---- sizes ----------------------------------------------------------------------------------------
struct EmbedPlan {
    int passes, digit, tile, tiles, piece, pieces;
    size_t key[2], pos[2], hist, part, shared, total;   // offsets in bytes
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
    // pieces of 8 tokens, of more where there would be over 2048 waves for them: few pieces leave the second kernel less to add (16384 tokens of
    // 2048 columns, a sixth of them one id's: 24.6 and 6 us of the two kernels with 512 pieces, 24.8 and 17 with 2048), too few leave the first
    // short of loads (65536 of 1024: 31 and 8 us with 512, 25 and 8 with 1024, 27 and 10 with 4096)
    const int64_t most = std::max((int64_t)512, 2048 / (((int64_t)dim + WAVE * 8 - 1) / (WAVE * 8)));
    p.piece = SPILL;
    while (((int64_t)tokens + p.piece - 1) / p.piece > most) p.piece *= 2;
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
    p.shared = take(((size_t)p.pieces + 1) * 4);
    return p;
}

template <typename E, typename T, typename I>
void embed_forward(const EmbedArgs& a, hipStream_t st)
{
    auto launch = [&](auto g) {
        constexpr int G = decltype(g)::value, SIDE = 256 / G;
        const int64_t n = ((int64_t)a.tokens + SIDE - 1) / SIDE;
        hipLaunchKernelGGL((embed_fwd_kernel<E, T, I, G>), dim3((unsigned)std::min(n, (int64_t)65536)), dim3(256), 0, st, a);
    };
    // as many lanes as a row has slices: a row takes two trips to memory, one behind the other, and short waves leave room for others' (a wave a row with four
    // slices a lane instead: 16384 rows of 2048 bf16 22.1 us against 20.9, of 8192 107 against 99; of 256 rows of 2048 3.5 against 2.5)
    if (a.dim <= 8 * 8) launch(std::integral_constant<int, 8>{});
    else if (a.dim <= 64 * 8) launch(std::integral_constant<int, 64>{});
    else if (a.dim <= 128 * 8) launch(std::integral_constant<int, 128>{});
    else launch(std::integral_constant<int, 256>{});
}
template <typename E, typename I, bool PAST>
void embed_sort(const EmbedArgs& a, bool place, dim3 grid, hipStream_t st)
{
    if (place) hipLaunchKernelGGL((embed_place_kernel<E, I, PAST>), grid, dim3(SORT_THREADS), 0, st, a);
    else hipLaunchKernelGGL((embed_count_kernel<E, I, PAST>), grid, dim3(SORT_THREADS), 0, st, a);
}
template <typename E, typename T, typename I>
void embed_backward(EmbedArgs a, char* ws, hipStream_t st)
{
    const EmbedPlan p = embed_plan(a.tokens, a.vocab, a.dim);
    const int64_t all = (int64_t)a.vocab * a.dim;
    // a tile alone needs no counts of others: a call of 1000 tokens of 512 columns and 5000 ids is ready for the next in 22 us of the host's time instead of 25
    const int turns = p.tiles == 1 ? 1 : 2, shares = a.tokens ? turns * p.passes : 1;
    a.hist = reinterpret_cast<int*>(ws + p.hist);
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.shared = reinterpret_cast<int*>(ws + p.shared);
    a.tile = p.tile; a.tiles = p.tiles; a.digit = p.digit;
    a.piece = p.piece; a.pieces = p.pieces;
    for (int k = 0; k < shares; ++k) {
        // shares of whole 16-byte words from the start
        a.fill_from = all / shares * k / 8 * 8;
        a.fill_to = k == shares - 1 ? all : all / shares * (k + 1) / 8 * 8;
        const int64_t fillers = (a.fill_to - a.fill_from) * (int64_t)sizeof(E) / (16 * SORT_THREADS * FILL_STORES) + 1;
        const dim3 grid((unsigned)(p.tiles + std::min(fillers, FILL_WORKGROUPS)));
        const int pass = k / turns, to = pass % 2;
        a.shift = pass * p.digit;
        a.key_in = pass ? reinterpret_cast<int*>(ws + p.key[1 - to]) : nullptr;
        a.pos_in = pass ? reinterpret_cast<int*>(ws + p.pos[1 - to]) : nullptr;
        a.key_out = reinterpret_cast<int*>(ws + p.key[to]);
        a.pos_out = reinterpret_cast<int*>(ws + p.pos[to]);
        if (all * (int64_t)sizeof(E) > STREAM_BYTES) embed_sort<E, I, true>(a, k % turns == turns - 1, grid, st);
        else embed_sort<E, I, false>(a, k % turns == turns - 1, grid, st);
    }
    if (!a.tokens) return;
    a.key = a.key_out;
    a.pos = a.pos_out;
    const unsigned slabs = (unsigned)((a.dim + WAVE * 8 - 1) / (WAVE * 8));
    hipLaunchKernelGGL((embed_sum_kernel<E, T>), dim3((unsigned)((p.pieces + 3) / 4), slabs), dim3(256), 0, st, a);
    if (p.pieces > 1)
        hipLaunchKernelGGL((embed_join_kernel<E>), dim3((unsigned)std::min(p.pieces - 1, JOIN_WORKGROUPS), slabs), dim3(JOIN_WAVES * WAVE), 0, st, a);
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
constexpr int32_t EMBED_WIDEST = 65535 * 512;           // columns that the workgroups along y of a launch reach

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
