// Rows brought to 8-bit integers: the scale of a row and the rounding of its values, as include/ss_quant.h defines them.
#pragma once
#include "ss_device.h"

namespace ss {

constexpr float Q_LEAST = 7.52316384526264e-37f;  // 2^-120
constexpr int Q_STEP = 128;                      // bytes of the contraction index that a step of a product takes: rows are a multiple of it
inline size_t quant_pitch(int32_t dim) { return dim < 1 ? 0 : ((size_t)dim + Q_STEP - 1) / Q_STEP * Q_STEP; }
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

}  // namespace ss
