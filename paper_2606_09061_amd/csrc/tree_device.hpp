// Helpers of libcptree's kernels and their launches.
#pragma once

#include "device.hpp"
#include "tree_attn.hpp"

namespace cptree {

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Launches with the rows in an argument block of their number's size: the full
// block costs the host 1.4 us more than a short one.
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

// The row whose workgroups item b belongs to: as many rows begin at or before
// it as lanes say so (every lane of a wave looks at two rows at most).
template <int N>
__device__ __forceinline__ TreeRow row_of(const RowsOf<TreeRow, N>& rows, int b) {
  static_assert(N <= 128, "two rows per lane");
  const int lane = threadIdx.x & 63;
  const bool lo = lane < N && rows.r[min(lane, N - 1)].item0 <= b;
  int n = __popcll(__builtin_amdgcn_ballot_w64(lo));
  if constexpr (N > 64) {
    const bool hi = 64 + lane < N && rows.r[min(64 + lane, N - 1)].item0 <= b;
    n += __popcll(__builtin_amdgcn_ballot_w64(hi));
  }
  return rows.r[__builtin_amdgcn_readfirstlane(n - 1)];
}

// Bit b: whether a node with this mask sees the key at offset o + b of its
// row's tree of n nodes (negative offsets are committed keys, o > -64).
__device__ __forceinline__ uint64_t seen64(const uint64_t* mask, int words, int n, int o) {
  if (o >= n) return 0;
  const int at = max(o, 0), w = at >> 6, sh = at & 63;
  uint64_t x = mask[w] >> sh;
  if (sh > 0 && w + 1 < words) x |= mask[w + 1] << (64 - sh);
  if (n - at < 64) x &= (1ull << (n - at)) - 1;
  return o >= 0 ? x : x << -o | ((1ull << -o) - 1);
}

// Whether a bf16 is an infinity or NaN, for both halves of a word.
__device__ __forceinline__ bool bad_lo(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool bad_hi(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }

// Takes the values that no product may meet out of one word of V, the keys at
// tree offsets k and k + 1: those past the row (k >= n), which may be
// anything, and infinities and NaN of the tree's own, of which bits 0 and 1 of
// the result tell.  Committed keys stay: every node sees them.
__device__ __forceinline__ uint32_t clean_word(uint32_t& w, int k, int n) {
  const bool lo = k >= 0 && bad_lo(w), hi = k + 1 >= 0 && bad_hi(w);
  if (lo || k >= n) w &= 0xffff0000u;
  if (hi || k + 1 >= n) w &= 0x0000ffffu;
  return (lo && k < n ? 1u : 0u) | (hi && k + 1 < n ? 2u : 0u);
}

// Notes in bad (a bit per node, LDS) the keys at tree offsets first + b for the
// bits b of `found`.
__device__ __forceinline__ void note_bad(unsigned long long* bad, uint32_t found, int first) {
  for (; found; found &= found - 1) {
    const int k = first + __ffs(found) - 1;
    atomicOr(&bad[k >> 6], 1ull << (k & 63));
  }
}

// What the infinite or NaN values of nodes in `bad` that a node with this mask
// sees add to feature d of its output.
template <int D, int B>
__device__ float bad_values(const unsigned long long* bad, const uint64_t* mask, int words,
                            const TreeRow& row, const AttnArgs& a, int kvh, int d) {
  const int32_t* bt_row = a.bt + (int64_t)row.req * a.mbr;
  float sum = 0.f;
  for (int w = 0; w < words; ++w)
    for (uint64_t x = bad[w] & mask[w]; x; x &= x - 1) {
      const int p = row.start + 64 * w + __ffsll((unsigned long long)x) - 1;
      const uint32_t v =
          a.v_cache[(((int64_t)bt_row[p / B] * a.hkv + kvh) * D + d) * B + p % B];
      if (bad_lo(v)) sum += __uint_as_float(v << 16);
    }
  return sum;
}

}  // namespace cptree
