// Slices of eight consecutive elements of rows of any length and alignment.
//
// A row's slices start at multiples of 8 elements.  The last one may reach up to 7 elements past the row: they belong to what
// stands behind it in the same tensor, but for the tensor's last row (`whole` false), whose last slice is read from further
// ahead, slice_limit, and shifted into place when it is used.  So a request is one access without a branch in every row, and no wave is
// slower than the others (read element by element, the last of 1536 bf16 rows of 4097 made a pass take 44 us instead of 22).
// Rows of less than 8 elements are read element by element; TINY: there may be such.
#pragma once
#include "ss_device.h"

namespace ss {

// Whether the slices of a row of n elements may reach past it.
__device__ __forceinline__ bool slice_whole(int n, bool last_row) { return n % 8 == 0 || (n >= 8 && !last_row); }
// Where the last request of a row starts.  Slices past it read there too.
__device__ __forceinline__ int slice_limit(int n, bool whole) { return whole ? (n - 1) / 8 * 8 : max(n - 8, 0); }
template <typename T, bool TINY>
__device__ __forceinline__ typename io8<T>::raw slice_request(const T* row, int t0, int n, int limit)
{
    if constexpr (TINY)
        if (n < 8) return io8<T>::template load<false>(row, max(min(n - t0, 8), 0));   // t0 is 0 or past the row
    return io8<T>::load_elem(row + min(t0, limit), 0u);
}
template <typename T>
__device__ __forceinline__ void slice_settle(typename io8<T>::raw& r, int t0, int n, int limit, bool whole)
{
    if (!whole && n >= 8) io8<T>::drop(r, max(t0 - limit, 0));
}
// the first n elements of the slice; none for n <= 0
template <typename T>
__device__ __forceinline__ void slice_store(T* row, int t0, int n, const float (&v)[8])
{
    if (n > 0) io8<T>::store_elem(row + t0, 0u, io8<T>::pack(v), n);
}


// Whether a result of so many bytes should go past the memory's cache (256 MB), as it could not be found there by who reads it, and would push out what is read
// next: 839 MB of logits' gradients behind their forward pass 472 -> 442 us for both, 419 MB of zeros before sums of 67 MB 160 -> 152.
constexpr int64_t STREAM_BYTES = (int64_t)128 << 20;

// whole slices at element alignment, past the caches
template <typename T>
__device__ __forceinline__ void store_past(T* p, u32x4 x)
{
    __builtin_nontemporal_store(x, reinterpret_cast<typename elem_aligned<u32x4, (int)sizeof(T)>::type*>(p));
}
// 16 bytes of T as numbers.  (A lane's store should be one of these, side by side with its neighbours': two past the caches from a lane, at every other 16 bytes
// each, took 155 us for 419 MB of float32 gradients; this takes 133, and stores through the caches 135, which cost who reads next 23.)
template <typename T> struct words16;
template <> struct words16<float> {
    static __device__ __forceinline__ void unpack(u32x4 x, float (&v)[4])
    {
        v[0] = __uint_as_float(x.x); v[1] = __uint_as_float(x.y); v[2] = __uint_as_float(x.z); v[3] = __uint_as_float(x.w);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[4])
    {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};
template <> struct words16<bf16_t> {
    static __device__ __forceinline__ void unpack(u32x4 x, float (&v)[8])
    {
        v[0] = bf16_lo(x.x); v[1] = bf16_hi(x.x); v[2] = bf16_lo(x.y); v[3] = bf16_hi(x.y);
        v[4] = bf16_lo(x.z); v[5] = bf16_hi(x.z); v[6] = bf16_lo(x.w); v[7] = bf16_hi(x.w);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[8])
    {
        return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
};

}  // namespace ss
