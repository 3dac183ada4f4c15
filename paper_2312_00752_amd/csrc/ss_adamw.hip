// A step of AdamW over many tensors at once, with moments in float32 or in 8 bits, for gfx950, with the C-ABI entry points (see
// include/ss_adamw.h).
//
// Every element is read and written once, 28 bytes of a float32 parameter with float32 moments and 16 with 8-bit ones, so a step is
// bound by HBM, and for small tensors by a launch.  The tensors' pointers travel in the kernel's arguments, as many as these hold, so nothing
// has to be copied to the device before; a workgroup finds the tensor that its chunk of elements belongs to.  A wave has 256 elements, a block of the
// 8-bit moments, four consecutive ones a lane.  The number of steps taken is read by all workgroups and counted by the last that ends.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>

#include "ss_adamw.h"
#include "ss_round8.h"

namespace ss {

constexpr int ADAMW_TENSORS = 48;      // of a launch: arguments have 4 KB
constexpr int ADAMW_THREADS = 256, ADAMW_STEP = ADAMW_THREADS * 4;   // elements of a workgroup and step
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

// four consecutive elements, of which n are there
__device__ __forceinline__ void load4(const void* p, bool low, int64_t i, int n, float (&v)[4])
{
    if (n >= 4) {
        if (low) {
            const u32x2v x = load_any<u32x2v>(static_cast<const bf16_t*>(p) + i, 0u);
            v[0] = bf16_lo(x.x); v[1] = bf16_hi(x.x); v[2] = bf16_lo(x.y); v[3] = bf16_hi(x.y);
        } else {
            const u32x4 x = load_any<u32x4>(static_cast<const float*>(p) + i, 0u);
            v[0] = __uint_as_float(x.x); v[1] = __uint_as_float(x.y); v[2] = __uint_as_float(x.z); v[3] = __uint_as_float(x.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = j >= n ? 0.0f : (low ? bf16_to_f32(static_cast<const bf16_t*>(p)[i + j]) : static_cast<const float*>(p)[i + j]);
    }
}
__device__ __forceinline__ void store4(void* p, bool low, int64_t i, int n, const float (&v)[4])
{
    if (n >= 4) {
        if (low) store_any(static_cast<bf16_t*>(p) + i, 0u, u32x2v{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
        else store_any(static_cast<float*>(p) + i, 0u, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) {
                if (low) static_cast<bf16_t*>(p)[i + j] = f32_to_io<bf16_t>(v[j]);
                else static_cast<float*>(p)[i + j] = v[j];
            }
    }
}
__device__ __forceinline__ uint32_t load_codes(const void* p, int64_t i, int n)
{
    const uint8_t* q = static_cast<const uint8_t*>(p) + i;
    if (n >= 4) return load_any<uint32_t>(q, 0u);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) w |= (uint32_t)q[j] << (8 * j);
    return w;
}
__device__ __forceinline__ void store_codes(void* p, int64_t i, int n, uint32_t w)
{
    uint8_t* q = static_cast<uint8_t*>(p) + i;
    if (n >= 4) {
        store_any(q, 0u, w);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) q[j] = (uint8_t)(w >> (8 * j));
}
template <bool SIGN>
__device__ __forceinline__ void decode(uint32_t codes, float scale, float (&v)[4])
{
    constexpr float top = SIGN ? 127.0f : 255.0f;
    const float c = scale * (1.0f / (top * top));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = SIGN ? (float)(int8_t)(codes >> (8 * j)) : (float)(uint8_t)(codes >> (8 * j));
        v[j] = q * fabsf(q) * c;
    }
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int s = 1; s < WAVE; s *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, s));
    return v;
}
// The codes of a wave's block, of which this lane has four values, and the block's scale.  turn: the first's place in the sequence, in 2^-32.
template <bool SIGN>
__device__ __forceinline__ uint32_t encode(const float (&v)[4], uint32_t turn, uint32_t apart, float& scale)
{
#pragma clang fp contract(off)
    constexpr float top = SIGN ? 127.0f : 255.0f;
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, magnitude(v[j]));
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
    const float unit = top * top * (1.0f / scale);
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float y = fabsf(v[j]) * unit, q = floorf(sqrtf(y));
        const float u = (float)((turn + j * apart) >> 8) * 0x1p-24f;
        int k = (int)fminf(q + (y - q * q > u * (2.0f * q + 1.0f) ? 1.0f : 0.0f), top);
        if (SIGN) k = v[j] < 0.0f ? -k : k;
        else k = v[j] > 0.0f ? max(k, 1) : 0;
        codes |= (uint32_t)(k & 255) << (8 * j);
    }
    return codes;
}

template <int BITS>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwArgs a)
{
#pragma clang fp contract(off)   // the moments are what the header's products and sums give, each rounded
    int k = 0, above = a.tensors;   // the tensor that has this chunk: start[k] <= blockIdx.x < start[above]
    while (above - k > 1) {
        const int mid = (k + above) / 2;
        if (a.start[mid] <= (int)blockIdx.x) k = mid;
        else above = mid;
    }
    const int taken = a.count[0];
    const uint32_t step = (uint32_t)taken + 1u;
    if (a.tensors > 0) {
        const AdamwTensor& e = a.tensor[k];
        const bool low_param = a.low_param[k], low_grad = a.low_grad[k];
        // 1 - beta^t = -expm1(t log beta)
        const float c1 = -expm1f((float)(step * a.log1)), c2 = -expm1f((float)(step * a.log2));
        const float lr = a.lr_device ? a.lr_device[0] : a.lr, gs = a.grad_scale ? a.grad_scale[0] : 1.0f;
        const float rate = lr / c1, root = 1.0f / sqrtf(c2), decay = lr * a.decay;
        const int64_t n = e.n, from = (int64_t)((int)blockIdx.x - a.start[k]) * a.chunk, to = min(from + a.chunk, n);
        for (int64_t i0 = from; i0 < to; i0 += ADAMW_STEP) {
            const int64_t i = i0 + threadIdx.x * 4;
            const int have = (int)max(min(n - i, (int64_t)4), (int64_t)0);
            float p[4], g[4], m[4], v[4], s[4];
            const int64_t block = (i0 + threadIdx.x / WAVE * 256) / SS_ADAMW_BLOCK;
            const bool there = block * SS_ADAMW_BLOCK < n;   // the same for a wave
            load4(low_param && e.master ? static_cast<const void*>(e.master) : e.param, low_param && !e.master, i, have, p);
            load4(e.grad, low_grad, i, have, g);
            if constexpr (BITS == 32) {
                load4(e.m, false, i, have, m);
                load4(e.v, false, i, have, v);
            } else {
                decode<true>(load_codes(e.m, i, have), there ? e.m_scale[block] : 0.0f, m);
                decode<false>(load_codes(e.v, i, have), there ? e.v_scale[block] : 0.0f, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= v[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[j] *= gs;
                m[j] = m[j] * a.beta1 + g[j] * a.rest1;
                v[j] = v[j] * a.beta2 + g[j] * g[j] * a.rest2;
                s[j] = sqrtf(v[j]);
                p[j] = fmaf(-decay, p[j], p[j]) - rate * (m[j] * __builtin_amdgcn_rcpf(fmaf(s[j], root, a.eps)));
            }
            if (low_param && e.master) store4(e.master, false, i, have, p);
            store4(e.param, low_param, i, have, p);
            if constexpr (BITS == 32) {
                store4(e.m, false, i, have, m);
                store4(e.v, false, i, have, v);
            } else {
                float ms, vs;
                const uint32_t at = (uint32_t)i;
                // behind the tensor's end m and s are 0
                store_codes(e.m, i, have, encode<true>(m, at * 0x6a09e667u + step * 0xbb67ae85u, 0x6a09e667u, ms));
                store_codes(e.v, i, have, encode<false>(s, at * 0x3c6ef372u + step * 0xa54ff53au, 0x3c6ef372u, vs));
                if (there && threadIdx.x % WAVE == 0) {
                    e.m_scale[block] = ms;
                    e.v_scale[block] = vs;
                }
            }
        }
    }
    if (!a.last) return;
    __syncthreads();   // all of the workgroup have read the count
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.count[1], 1) == (int)gridDim.x - 1) {
            a.count[1] = 0;
            a.count[0] = taken + 1;
        }
    }
}

template <bool SIGN, typename T>
__global__ __launch_bounds__(256) void adamw_values_kernel(const void* codes, const float* scale, T* out, int64_t n)
{
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        const int have = (int)min(n - i, (int64_t)4);
        float v[4];
        decode<SIGN>(load_codes(codes, i, have), scale[i / SS_ADAMW_BLOCK], v);
        store4(out, sizeof(T) == 2, i, have, v);
    }
}

}  // namespace ss

namespace {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool known(int32_t dtype) { return dtype == SS_F32 || dtype == SS_BF16; }
inline size_t bytes_of(int32_t dtype) { return dtype == SS_BF16 ? 2 : 4; }
constexpr int64_t ADAMW_MOST = (int64_t)1 << 40;           // elements of a tensor
constexpr int64_t ADAMW_CHUNKS = ((int64_t)1 << 24) - 1;   // of a launch: it has fewer than 2^32 threads

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
    if (!p->lr_device && !some(p->lr)) return SS_ERR_UNSUPPORTED;
    const bool eight = p->state_bits == 8;
    int64_t all = 0;
    for (int k = 0; k < p->tensors; ++k) {
        const int rc = check_tensor(p->list[k], eight);
        if (rc != SS_OK) return rc;
        all += p->list[k].n;
    }
    ss::AdamwArgs a{};
    a.count = p->count;
    a.lr = (float)p->lr; a.eps = (float)p->eps; a.decay = (float)p->weight_decay;
    a.beta1 = (float)p->beta1; a.rest1 = (float)(1.0 - p->beta1);
    a.beta2 = (float)p->beta2; a.rest2 = (float)(1.0 - p->beta2);
    a.log1 = std::log(p->beta1); a.log2 = std::log(p->beta2);
    a.lr_device = p->lr_device; a.grad_scale = p->grad_scale;
    // a step a chunk while that gives few workgroups, up to eight
    int64_t chunk = std::min(std::max(all / (ss::ADAMW_STEP * (int64_t)4096), (int64_t)1), (int64_t)8) * ss::ADAMW_STEP;
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
        if (eight) hipLaunchKernelGGL(ss::adamw_kernel<8>, grid, dim3(ss::ADAMW_THREADS), 0, st, a);
        else hipLaunchKernelGGL(ss::adamw_kernel<32>, grid, dim3(ss::ADAMW_THREADS), 0, st, a);
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
    const dim3 grid((unsigned)std::min((p->n + 1023) / 1024, (int64_t)65536));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto t) {
        typedef decltype(t) T;
        if (p->with_sign) hipLaunchKernelGGL((ss::adamw_values_kernel<true, T>), grid, dim3(256), 0, st, p->codes, p->scale, static_cast<T*>(p->out), p->n);
        else hipLaunchKernelGGL((ss::adamw_values_kernel<false, T>), grid, dim3(256), 0, st, p->codes, p->scale, static_cast<T*>(p->out), p->n);
    };
    if (p->out_dtype == SS_F32) launch(float());
    else launch(ss::bf16_t());
    return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_LAUNCH;
}

}  // extern "C"
