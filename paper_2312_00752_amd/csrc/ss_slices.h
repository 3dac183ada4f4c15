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

}  // namespace ss
