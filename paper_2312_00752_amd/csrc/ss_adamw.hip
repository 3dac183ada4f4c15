// A step of AdamW over many tensors at once, with moments in float32 or in 8 bits, for gfx950, with the C-ABI entry points (see
// include/ss_adamw.h).
//
// Every element is read and written once, 28 bytes of a float32 parameter with float32 moments and 16 with 8-bit ones, so a step is
// bound by HBM (67 million float32 350 us, 5.4 TB/s; 126 million bf16 with float32 copies and 8-bit moments 356 us, 5.7 TB/s), and for small
// tensors by a launch (0.2 million elements in 16 tensors 4.9 us).  The tensors' pointers travel in the kernel's arguments, as many as these hold, so
// nothing has to be copied to the device before; a workgroup finds the tensor that its chunk of elements belongs to.  A wave has 256 elements, a
// block of the 8-bit moments, four consecutive ones a lane.  The number of steps taken is read by all workgroups and counted by the last to say so.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ss_adamw.h"
#include "ss_round8.h"
#include "ss_slices.h"

namespace ss {

constexpr int ADAMW_TENSORS = 48;      // of a launch: arguments have 4 KB
constexpr float ADAMW_LEAST = 7.88860905e-31f;   // 2^-100

struct AdamwTensor {
    int64_t n;
    void* param;
    const void* grad;
    float* master;
    void *m, *v;
    float *m_scale, *v_scale;
};
struct AdamwArgs {
    AdamwTensor tensor[ADAMW_TENSORS];
    int start[ADAMW_TENSORS + 1];      // the first chunk of each; behind the last, all of them
    uint8_t low_param[ADAMW_TENSORS], low_grad[ADAMW_TENSORS];
    int tensors, chunk, last;          // elements of a chunk; whether this is the call's last launch
    int* count;
    float lr, beta1, rest1, beta2, rest2, eps, decay;
    double log1, log2;                 // natural logarithms of the betas (-infinity for 0)
    const float *lr_device, *grad_scale;
};

// ---- four consecutive elements of a lane, of which n are there (FULL: all) ---------------------------
template <bool FULL, typename T>
__device__ __forceinline__ void load4(const T* p, int n, float (&v)[4])
{
    if (FULL || n >= 4) {
        if constexpr (sizeof(T) == 2) {
            const u32x2v x = load_any<u32x2v>(p, 0u);
            v[0] = bf16_lo(x.x); v[1] = bf16_hi(x.x); v[2] = bf16_lo(x.y); v[3] = bf16_hi(x.y);
        } else {
            const u32x4 x = load_any<u32x4>(p, 0u);
            v[0] = __uint_as_float(x.x); v[1] = __uint_as_float(x.y); v[2] = __uint_as_float(x.z); v[3] = __uint_as_float(x.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < n ? io_to_f32<T>(p[j]) : 0.0f;
    }
}
template <bool FULL, typename T>
__device__ __forceinline__ void store4(T* p, int n, const float (&v)[4])
{
    if (FULL || n >= 4) {
        if constexpr (sizeof(T) == 2) store_any(p, 0u, u32x2v{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
        else store_any(p, 0u, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = f32_to_io<T>(v[j]);
    }
}
template <bool FULL>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* q, int n)
{
    if (FULL || n >= 4) return load_any<uint32_t>(q, 0u);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) w |= (uint32_t)q[j] << (8 * j);
    return w;
}
template <bool FULL>
__device__ __forceinline__ void store_codes(uint8_t* q, int n, uint32_t w)
{
    if (FULL || n >= 4) {
        store_any(q, 0u, w);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) q[j] = (uint8_t)(w >> (8 * j));
}

// ---- moments in 8 bits ------------------------------------------------------------------------------
template <bool SIGN>
__device__ __forceinline__ void decode(uint32_t codes, float scale, float (&v)[4])
{
    constexpr float top = SIGN ? 127.0f : 255.0f;
    const float c = scale * (1.0f / (top * top));
    if (SIGN) codes ^= 0x80808080u;   // 128 more, without a sign
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = (float)(codes >> (8 * j) & 255u) - (SIGN ? 128.0f : 0.0f);
        v[j] = q * fabsf(q) * c;
    }
}
// The largest of a wave's values in all of its lanes, by the vector unit's own exchanges: lanes of rows of 16, then the rows.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#define SS_MAX_FROM(control, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, control, rows, 0xf, false))
    SS_MAX_FROM(0x111, 0xf);   // the lane one before, two, four, eight
    SS_MAX_FROM(0x112, 0xf);
    SS_MAX_FROM(0x114, 0xf);
    SS_MAX_FROM(0x118, 0xf);
    SS_MAX_FROM(0x142, 0xa);   // the last lane of the row before, into the second and fourth row
    SS_MAX_FROM(0x143, 0xc);   // the last of the first half, into the second
#undef SS_MAX_FROM
    return (uint32_t)__builtin_amdgcn_readlane((int)v, WAVE - 1);
}
// Correctly rounded from 2^-100 on: the hardware's root is off by a unit in the last place at most, and a step of Newton's method from there
// has an exact residual.  (The compiler's own takes twice as many instructions; the step of 126 million parameters was bound by them.)
__device__ __forceinline__ float root_of(float v)
{
    const float s = __builtin_amdgcn_sqrtf(v), h = 0.5f * __builtin_amdgcn_rcpf(s);
    return s > 0.0f && s < INFINITY ? fmaf(fmaf(-s, s, v), h, s) : s;
}
// The codes of a wave's block, of which this lane has four values, and the block's scale.  turn: the first's place in the sequence, in 2^-32.
// q is the floor of the hardware's root of y: where y is so near a square that it is one off, the code is the same.
template <bool SIGN>
__device__ __forceinline__ uint32_t encode(const float (&v)[4], uint32_t turn, uint32_t apart, float& scale)
{
    constexpr float top = SIGN ? 127.0f : 255.0f;
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, SIGN ? magnitude(v[j]) : __float_as_uint(v[j]));
    most = wave_max(most);
    scale = __uint_as_float(most);
    if (most >= 0x7f800000u) {
        scale = __uint_as_float(0x7fc00000u);
        return 0u;
    }
    if (scale < ADAMW_LEAST) {
        scale = 0.0f;
        return 0u;
    }
    // 1 / scale, correctly rounded as root_of is
    const float r0 = __builtin_amdgcn_rcpf(scale), unit = top * top * fmaf(fmaf(-scale, r0, 1.0f), r0, r0);
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float y = fabsf(v[j]) * unit;
        q[j] = floorf(__builtin_amdgcn_sqrtf(y));
        const float u = (float)((turn + j * apart) >> 8);   // in 2^-24, and 2 q + 1 in 2^24
        const float apart_by = u * fmaf(q[j], 0x1p-23f, 0x1p-24f);
        q[j] = fminf(q[j] + (fmaf(-q[j], q[j], y) > apart_by ? 1.0f : 0.0f), top);
        if (!SIGN) q[j] = fmaxf(q[j], v[j] > 0.0f ? 1.0f : 0.0f);
    }
    // whole numbers, as the low bytes of floats that have no bits below one
    constexpr float up = 12582912.0f;
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = __float_as_uint((SIGN ? copysignf(q[j], v[j]) : q[j]) + up);
    return __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) | __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
}

// ---- a step -------------------------------------------------------------------------------------------
struct StepFactors {
    float rate, root, decay, scale;   // of the moments' quotient, of sqrt(v), of the parameter, of the gradient
    uint32_t step;
};
// A workgroup's chunk of a tensor, from element `from` on.  P: the parameter's type; MASTER: its float32 copy is updated; R: the gradient's.
template <int BITS, int THREADS, typename P, bool MASTER, typename R, bool FULL>
__device__ __forceinline__ void adamw_chunk(const AdamwArgs& a, const AdamwTensor& e, int64_t from, int n, const StepFactors& f)
{
#pragma clang fp contract(off)   // the moments are what the header's products and sums give, each rounded
    P* const param = static_cast<P*>(e.param) + from;
    const R* const grad = static_cast<const R*>(e.grad) + from;
    float* const master = MASTER ? e.master + from : nullptr;
    for (int i0 = 0; i0 < n; i0 += THREADS * 4) {
        const int i = i0 + threadIdx.x * 4, have = FULL ? 4 : max(min(n - i, 4), 0);
        float p[4], g[4], m[4], v[4], s[4];
        if constexpr (MASTER) load4<FULL>(master + i, have, p);
        else load4<FULL>(param + i, have, p);
        load4<FULL>(grad + i, have, g);
        const int block = (i0 + threadIdx.x / WAVE * 256) / SS_ADAMW_BLOCK;
        const bool there = FULL || block * SS_ADAMW_BLOCK < n;   // the same for a wave
        float *const m_scale = BITS == 8 ? e.m_scale + from / SS_ADAMW_BLOCK + block : nullptr, *const v_scale = BITS == 8 ? e.v_scale + from / SS_ADAMW_BLOCK + block : nullptr;
        if constexpr (BITS == 32) {
            load4<FULL>(static_cast<const float*>(e.m) + from + i, have, m);
            load4<FULL>(static_cast<const float*>(e.v) + from + i, have, v);
        } else {
            const uint32_t cm = load_codes<FULL>(static_cast<const uint8_t*>(e.m) + from + i, have), cv = load_codes<FULL>(static_cast<const uint8_t*>(e.v) + from + i, have);
            const float am = there ? *m_scale : 0.0f, av = there ? *v_scale : 0.0f;
            decode<true>(cm, am, m);
            decode<false>(cv, av, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= v[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] *= f.scale;
            m[j] = m[j] * a.beta1 + g[j] * a.rest1;
            v[j] = v[j] * a.beta2 + g[j] * g[j] * a.rest2;
            s[j] = root_of(v[j]);
        }
        // below 2^-100 the residual of the root is no normal number, and below 2^-126 neither is v, whose
        // root the hardware takes as 0 (a step of m / eps: 10^10 for a gradient of 1e-18 and eps of 1e-30)
        if (fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < 0x1p-100f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = v[j] < 0x1p-100f ? root_of(v[j] * 0x1p64f) * 0x1p-32f : s[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p[j] = fmaf(-f.rate, m[j] * __builtin_amdgcn_rcpf(fmaf(s[j], f.root, a.eps)), fmaf(-f.decay, p[j], p[j]));
        }
        if constexpr (MASTER) store4<FULL>(master + i, have, p);
        store4<FULL>(param + i, have, p);
        if constexpr (BITS == 32) {
            store4<FULL>(static_cast<float*>(e.m) + from + i, have, m);
            store4<FULL>(static_cast<float*>(e.v) + from + i, have, v);
        } else {
            float am, av;
            const uint32_t at = (uint32_t)(from + i);
            // behind the tensor's end m and s are 0
            store_codes<FULL>(static_cast<uint8_t*>(e.m) + from + i, have, encode<true>(m, at * 0x6a09e667u + f.step * 0xbb67ae85u, 0x6a09e667u, am));
            store_codes<FULL>(static_cast<uint8_t*>(e.v) + from + i, have, encode<false>(s, at * 0x3c6ef372u + f.step * 0xa54ff53au, 0x3c6ef372u, av));
            if (there && threadIdx.x % WAVE == 0) {
                *m_scale = am;
                *v_scale = av;
            }
        }
    }
}
template <int BITS, int THREADS, typename P, bool MASTER, typename R>
__device__ __forceinline__ void adamw_chunk_of(const AdamwArgs& a, const AdamwTensor& e, int64_t from, int n, const StepFactors& f)
{
    if (n % (THREADS * 4) == 0) adamw_chunk<BITS, THREADS, P, MASTER, R, true>(a, e, from, n, f);
    else adamw_chunk<BITS, THREADS, P, MASTER, R, false>(a, e, from, n, f);
}

template <int BITS, int THREADS>
__global__ __launch_bounds__(THREADS) void adamw_kernel(const AdamwArgs a)
{
    const int taken = __builtin_amdgcn_readfirstlane(a.count[0]);
    int k = 0, above = a.tensors;   // the tensor that has this chunk: start[k] <= blockIdx.x < start[above]
    while (above - k > 1) {
        const int mid = (k + above) / 2;
        if (a.start[mid] <= (int)blockIdx.x) k = mid;
        else above = mid;
    }
    if (a.last) {
        asm volatile("" ::"s"(taken));   // has arrived
        __syncthreads();                  // all of the workgroup have read the count; the last workgroup that says so writes it
    }
    // A workgroup's word costs 13 ns, one behind the other: said first where each has one step to do (the others wait for memory meanwhile), else
    // last, when they no longer stand in a queue (16 million elements, 8 bits, in 2048 workgroups: 45 us against 65 with the word first).
    auto say = [&]() {
        if (threadIdx.x == 0 && atomicAdd(&a.count[1], 1) == (int)gridDim.x - 1) {
            a.count[1] = 0;
            a.count[0] = taken + 1;
        }
    };
    const bool first = a.chunk == THREADS * 4 || a.tensors == 0;
    if (a.last && first) say();
    if (a.tensors == 0) return;
    StepFactors f;
    f.step = (uint32_t)taken + 1u;
    // 1 - beta^t = -expm1(t log beta)
    const float c1 = -expm1f((float)(f.step * a.log1)), c2 = -expm1f((float)(f.step * a.log2));
    const float lr = a.lr_device ? a.lr_device[0] : a.lr;
    f.rate = lr / c1;
    f.root = 1.0f / sqrtf(c2);
    f.decay = lr * a.decay;
    f.scale = a.grad_scale ? a.grad_scale[0] : 1.0f;
    const AdamwTensor& e = a.tensor[k];
    const int64_t from = (int64_t)((int)blockIdx.x - a.start[k]) * a.chunk;
    const int n = (int)min((int64_t)a.chunk, e.n - from);
    if (a.low_grad[k]) {
        if (!a.low_param[k]) adamw_chunk_of<BITS, THREADS, float, false, bf16_t>(a, e, from, n, f);
        else if (e.master) adamw_chunk_of<BITS, THREADS, bf16_t, true, bf16_t>(a, e, from, n, f);
        else adamw_chunk_of<BITS, THREADS, bf16_t, false, bf16_t>(a, e, from, n, f);
    } else {
        if (!a.low_param[k]) adamw_chunk_of<BITS, THREADS, float, false, float>(a, e, from, n, f);
        else if (e.master) adamw_chunk_of<BITS, THREADS, bf16_t, true, float>(a, e, from, n, f);
        else adamw_chunk_of<BITS, THREADS, bf16_t, false, float>(a, e, from, n, f);
    }
    if (a.last && !first) say();
}

// 16 bytes of the result a lane.  PAST: it goes past the caches.  Bound by HBM: 126 million bf16 (378 MB) 58 us, 6.5 TB/s (65 through the
// caches; behind a step 70).
template <bool SIGN, typename T, bool PAST>
__global__ __launch_bounds__(256) void adamw_values_kernel(const void* codes, const float* scale, T* out, int64_t n)
{
    constexpr int N = 16 / sizeof(T);
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N; i < n; i += (int64_t)gridDim.x * 256 * N) {
        const uint8_t* q = static_cast<const uint8_t*>(codes) + i;
        const int have = (int)min(n - i, (int64_t)N);
        const float s = scale[i / SS_ADAMW_BLOCK];
        float v[N / 4][4];
        if (have == N) {
            uint32_t c[N / 4];
            if constexpr (N == 8) {
                const u32x2v w = load_any<u32x2v>(q, 0u);
                c[0] = w.x;
                c[1] = w.y;
            } else {
                c[0] = load_any<uint32_t>(q, 0u);
            }
#pragma unroll
            for (int k = 0; k < N / 4; ++k) decode<SIGN>(c[k], s, v[k]);
            u32x4 x;
            if constexpr (N == 8) x = u32x4{pack_bf16x2(v[0][0], v[0][1]), pack_bf16x2(v[0][2], v[0][3]), pack_bf16x2(v[1][0], v[1][1]), pack_bf16x2(v[1][2], v[1][3])};
            else x = words16<float>::pack(v[0]);
            if constexpr (PAST) store_past(out + i, x);
            else store_any(out + i, 0u, x);
        } else {
#pragma unroll
            for (int k = 0; k < N / 4; ++k) {
                decode<SIGN>(load_codes<false>(q + 4 * k, have - 4 * k), s, v[k]);
                store4<false>(out + i + 4 * k, have - 4 * k, v[k]);
            }
        }
    }
}

}  // namespace ss

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool known(int32_t dtype) { return dtype == SS_F32 || dtype == SS_BF16; }
inline size_t bytes_of(int32_t dtype) { return dtype == SS_BF16 ? 2 : 4; }
constexpr int64_t ADAMW_MOST = (int64_t)1 << 40;           // elements of a tensor
constexpr int64_t ADAMW_CHUNKS = ((int64_t)1 << 22) - 1;   // of a launch: it has fewer than 2^32 threads

int check_tensor(const ss_adamw_tensor& t, bool eight)
{
    if (t.n < 0) return SS_ERR_SHAPE;
    if (!known(t.param_dtype) || !known(t.grad_dtype) || t.n > ADAMW_MOST) return SS_ERR_UNSUPPORTED;
    if (t.master && t.param_dtype != SS_BF16) return SS_ERR_UNSUPPORTED;
    if (t.n == 0) return SS_OK;
    if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return SS_ERR_NULL;
    if (!aligned_to(t.param, bytes_of(t.param_dtype)) || !aligned_to(t.grad, bytes_of(t.grad_dtype)) || !aligned_to(t.master, 4)) return SS_ERR_ALIGN;
    if (eight ? !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4) : !aligned_to(t.m, 4) || !aligned_to(t.v, 4)) return SS_ERR_ALIGN;
    return SS_OK;
}
inline bool some(double v) { return v >= 0.0 && std::isfinite((float)v); }

}  // namespace

extern "C" {

int ss_adamw_step(const ss_adamw_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    if (p->tensors < 0) return SS_ERR_SHAPE;
    if (p->state_bits != 32 && p->state_bits != 8) return SS_ERR_UNSUPPORTED;
    if (!p->count || (p->tensors > 0 && !p->list)) return SS_ERR_NULL;
    if (!aligned_to(p->count, 4) || !aligned_to(p->lr_device, 4) || !aligned_to(p->grad_scale, 4)) return SS_ERR_ALIGN;
    if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0) || !some(p->eps) || !some(p->weight_decay)) return SS_ERR_UNSUPPORTED;
    if (p->eps != 0.0 && p->eps < 0x1p-126) return SS_ERR_UNSUPPORTED;   // the reciprocal of no normal number is infinite: 0 / eps would be NaN
    if (!p->lr_device && !some(p->lr)) return SS_ERR_UNSUPPORTED;
    const bool eight = p->state_bits == 8;
    int64_t all = 0, small = 0;   // elements; workgroups of 256 threads for them
    for (int k = 0; k < p->tensors; ++k) {
        const int rc = check_tensor(p->list[k], eight);
        if (rc != SS_OK) return rc;
        all += p->list[k].n;
        small += (p->list[k].n + 1023) / 1024;
    }
    ss::AdamwArgs a{};
    a.count = p->count;
    a.lr = (float)p->lr; a.eps = (float)p->eps; a.decay = (float)p->weight_decay;
    a.beta1 = (float)p->beta1; a.rest1 = (float)(1.0 - p->beta1);
    a.beta2 = (float)p->beta2; a.rest2 = (float)(1.0 - p->beta2);
    a.log1 = std::log(p->beta1); a.log2 = std::log(p->beta2);
    a.lr_device = p->lr_device; a.grad_scale = p->grad_scale;
    // Few workgroups, for the sake of their words: of 256, 512 or 1024 threads, and 256 of the last, more only where each has two steps.  Float32 in us with
    // 256 / 512 / 1024 threads: 65536 elements 4.3 / 4.4 / 5.0; 262144 6.2 / 5.0 / 5.2; 2 million 12.3 / 11.2 / 10.2; 67 million 357 / 356 / 350;
    // 8 bits 5.0 / 5.7 / 6.3; 7.0 / 6.3 / 6.8; 14.2 / 13.6 / 11.6; 214 / 208 / 201.
    const int threads = small <= 64 ? 256 : (small <= 512 ? 512 : 1024), each = threads * 4;
    int64_t chunk = std::min(all / (each * (int64_t)256) + 1, (int64_t)(8192 / each)) * each;
    while (all / chunk > ADAMW_CHUNKS - ss::ADAMW_TENSORS && chunk < (1 << 30)) chunk *= 2;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    int k = 0;
    do {
        // as many tensors as the arguments hold, and their chunks a launch; one tensor's may need larger ones
        int64_t chunks = 0;
        a.tensors = 0;
        while (k < p->tensors && a.tensors < ss::ADAMW_TENSORS) {
            const ss_adamw_tensor& t = p->list[k];
            int64_t size = chunk;
            if (a.tensors == 0)
                while ((t.n + size - 1) / size > ADAMW_CHUNKS) size *= 2;
            const int64_t more = (t.n + size - 1) / size;
            if (t.n == 0) {
                ++k;
                continue;
            }
            if (a.tensors > 0 && (chunks + more > ADAMW_CHUNKS || a.chunk != chunk)) break;
            a.chunk = (int)size;
            a.tensor[a.tensors] = {t.n, t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale};
            a.low_param[a.tensors] = t.param_dtype == SS_BF16;
            a.low_grad[a.tensors] = t.grad_dtype == SS_BF16;
            a.start[a.tensors++] = (int)chunks;
            chunks += more;
            ++k;
        }
        a.start[a.tensors] = (int)chunks;
        while (k < p->tensors && p->list[k].n == 0) ++k;
        a.last = k == p->tensors;
        const dim3 grid((unsigned)std::max(chunks, (int64_t)1));
        auto launch = [&](auto n) {
            constexpr int THREADS = decltype(n)::value;
            if (eight) hipLaunchKernelGGL((ss::adamw_kernel<8, THREADS>), grid, dim3(THREADS), 0, st, a);
            else hipLaunchKernelGGL((ss::adamw_kernel<32, THREADS>), grid, dim3(THREADS), 0, st, a);
        };
        if (threads == 256) launch(std::integral_constant<int, 256>());
        else if (threads == 512) launch(std::integral_constant<int, 512>());
        else launch(std::integral_constant<int, 1024>());
    } while (!a.last);
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

int ss_adamw_values(const ss_adamw_values_params* p, void* stream)
{
    if (!p) return SS_ERR_NULL;
    if (p->n < 0) return SS_ERR_SHAPE;
    if (!known(p->out_dtype) || p->n > ADAMW_MOST || (p->with_sign & ~1)) return SS_ERR_UNSUPPORTED;
    if (p->n == 0) return SS_OK;
    if (!p->codes || !p->scale || !p->out) return SS_ERR_NULL;
    if (!aligned_to(p->scale, 4) || !aligned_to(p->out, bytes_of(p->out_dtype))) return SS_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto with = [&](auto t, auto past) {
        typedef decltype(t) T;
        constexpr bool PAST = decltype(past)::value;
        constexpr int64_t EACH = 256 * 16 / sizeof(T);
        const dim3 grid((unsigned)std::min((p->n + EACH - 1) / EACH, (int64_t)65536));
        if (p->with_sign) hipLaunchKernelGGL((ss::adamw_values_kernel<true, T, PAST>), grid, dim3(256), 0, st, p->codes, p->scale, static_cast<T*>(p->out), p->n);
        else hipLaunchKernelGGL((ss::adamw_values_kernel<false, T, PAST>), grid, dim3(256), 0, st, p->codes, p->scale, static_cast<T*>(p->out), p->n);
    };
    auto launch = [&](auto t) {
        if (p->n * (int64_t)sizeof(t) > ss::STREAM_BYTES) with(t, std::true_type());
        else with(t, std::false_type());
    };
    if (p->out_dtype == SS_F32) launch(float());
    else launch(ss::bf16_t());
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
