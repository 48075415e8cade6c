// q8_rows.cuh -- how the rows of the 8-bit norm lie and what of them is read at one time: index
// arithmetic alone (norm_q8.cu), so that it can be checked on the host.
#pragma once

namespace rdn {

// How a row lies: its rows on 16 bytes (kVectors); every row the same number of elements behind a group of 8 on
// 16 bytes in all operands, as rows of an odd length one after the other are (kShifted: the groups inside the
// row in vectors, the two at its ends, which its neighbours share, element by element); or neither.
enum Lie { kSingle, kShifted, kVectors };

// Lane t's group n of a row of D that is `off` elements behind: the row's elements i.. i + 7.
template <int kLie>
__host__ __device__ __forceinline__ int place(int n, int t, int lanes, int off) {
  return (n * lanes + t) * 8 - (kLie == kShifted ? off : 0);
}
template <int kLie>
__host__ __device__ __forceinline__ bool whole(int i, int D) {
  return kLie == kVectors ? i < D : kLie == kShifted && i >= 0 && i + 8 <= D;
}

// How the group from element i of a row on is read: not at all, element by element, or as 8 elements at once,
// those outside the row among them (they are its neighbours', or lie between two rows).
enum Read { kNothing, kElements, kGroup };
// (near_end: the row is one of the tensor's last near_end_rows(D))
template <int kLie>
__host__ __device__ __forceinline__ Read read_of(int i, int D, bool near_end) {
  if (kLie == kVectors) return i < D ? kGroup : kNothing;
  if (i >= D || i <= -8) return kNothing;
  return kLie == kShifted && (i + 8 <= D || !near_end) ? kGroup : kElements;
}
// A group that starts in a row ends at most 7 elements behind it.  The rows that follow it have D elements each, so
// that those with fewer than 7 of them behind are the last 7 / D, rounded up.
__host__ __device__ __forceinline__ int near_end_rows(int D) { return D >= 7 ? 1 : (7 + D - 1) / D; }

}  // namespace rdn
