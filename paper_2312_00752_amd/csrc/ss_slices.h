// Slices of eight consecutive elements of rows of any length and alignment.
//
// A row's slices start at multiples of 8 elements.  The last one may reach up to 7 elements past the row: they belong to what
// stands behind it in the same tensor, but for the tensor's last row (and rows of less than 8 elements), whose slices are
// read element by element (`whole` false).
#pragma once
#include "ss_device.h"

namespace ss {

template <typename T>
__device__ __forceinline__ typename io8<T>::raw slice_load(const T* row, int t0, int n, bool whole)   // n: elements of the row
{
    if (whole) return io8<T>::load_elem(row + t0, 0u);
    return io8<T>::template load<false>(row + t0, min(8, n - t0));
}
// the first n elements of the slice; none for n <= 0
template <typename T>
__device__ __forceinline__ void slice_store(T* row, int t0, int n, const float (&v)[8])
{
    if (n > 0) io8<T>::store_elem(row + t0, 0u, io8<T>::pack(v), n);
}

}  // namespace ss
