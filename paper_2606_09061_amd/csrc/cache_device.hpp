// Helpers of libcpcache's kernels and their launches.
#pragma once

#include "cache_kernels.hpp"
#include "device.hpp"

namespace cpcache {

// Launches with the rows in an argument block of their number's size: the full
// block costs the host more than a short one.
template <class T, int N, class F>
hipError_t by_size(const RowsOf<T, N>& rows, int n, F&& launch) {
  if (n <= kFewRows) {
    RowsOf<T, kFewRows> few;
    for (int i = 0; i < kFewRows; ++i) few.r[i] = rows.r[i];  // with the places behind the rows
    launch(few);
  } else {
    launch(rows);
  }
  return hipGetLastError();
}

template <class F>
hipError_t by_size(const AttnBatch& b, int n_groups, int n_rows, F&& launch) {
  if (n_rows <= kFewRows && n_groups <= 4) {
    FewAttnBatch few;
    for (int i = 0; i < 4; ++i) few.g[i] = b.g[i];
    for (int i = 0; i <= kFewRows; ++i) few.r[i] = b.r[i];
    launch(few);
  } else {
    launch(b);
  }
  return hipGetLastError();
}

// The index of the row that item b belongs to, the last whose first item is at
// or before it; uniform over the wave, whose lanes look at N / 64 rows each.
// `at` is the member that holds a row's first item.
template <class T, int N>
__device__ __forceinline__ int row_index(const T (&rows)[N], int32_t T::*at, int b) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int r0 = 0; r0 < N; r0 += 64) {
    const bool mine = r0 + lane < N && rows[r0 + lane < N ? r0 + lane : N - 1].*at <= b;
    n += __popcll(__builtin_amdgcn_ballot_w64(mine));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

}  // namespace cpcache
