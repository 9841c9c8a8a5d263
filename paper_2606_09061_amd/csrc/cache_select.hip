// Selection of pages by the bounds of their keys (include/cp_cache.h).
//
// The score of a page is the largest product that a key within its bounds can
// have with one of a group's q heads.  Which pages are selected hangs on the
// order of the scores, so they are fp64: products of bf16 are exact in it and
// their sums are, for all but extreme values, too, whatever their order.
#include "cache_device.hpp"

namespace cpcache {

using cpattn::bf16hi;
using cpattn::bf16lo;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Order-preserving keys of scores: NaN above all numbers, -0 as +0.
constexpr uint64_t kNanKey = ~0ull - 1, kForcedKey = ~0ull;
__device__ __forceinline__ uint64_t key_of(double x) {
  if (x != x) return kNanKey;
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}

template <int Bit>
__device__ __forceinline__ uint64_t partner64(uint64_t x) {
  const float lo = cpattn::lane_partner<Bit>(__uint_as_float((uint32_t)x));
  const float hi = cpattn::lane_partner<Bit>(__uint_as_float((uint32_t)(x >> 32)));
  return (uint64_t)__float_as_uint(lo) | (uint64_t)__float_as_uint(hi) << 32;
}

// One step of a sum over lanes that differ in `Bit`: while a lane holds more than
// one head's sum, each side keeps half of them and gives away the others.
template <int Bit, int N, int G>
__device__ __forceinline__ void sum_step(double (&u)[G], int lane) {
  if constexpr (N > 1) {
    const bool up = lane & Bit;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const double keep = up ? u[e + N / 2] : u[e], give = up ? u[e] : u[e + N / 2];
      u[e] = keep + __longlong_as_double((long long)partner64<Bit>(
                        (uint64_t)__double_as_longlong(give)));
    }
  } else {
    u[0] += __longlong_as_double((long long)partner64<Bit>((uint64_t)__double_as_longlong(u[0])));
  }
}

template <int Bit>
__device__ __forceinline__ uint64_t max_step(uint64_t k) {
  const uint64_t o = partner64<Bit>(k);
  return o > k ? o : k;
}

// Scores.  A workgroup takes kScorePages pages of one (token, kv head), its waves
// 64 / L of them at a time, L = D / 8 lanes a page with 8 features each.  With
// lo + hi and hi - lo of a feature, 2 max(q lo, q hi) = q (lo + hi) + |q| (hi - lo):
// two fp64 multiply-adds per head and feature, which with the conversions are
// 14 fp64-rate operations per 4 bytes of bounds at 4 heads a group; the bounds'
// stream is as long.
template <int D, int G, class Rows>
__global__ __launch_bounds__(kThreads) void score_kernel(const Rows rows, const SelectArgs a,
                                                         const uint16_t* __restrict__ q,
                                                         const uint4* __restrict__ bounds,
                                                         const int32_t* __restrict__ bt,
                                                         uint64_t* __restrict__ scores) {
  constexpr int L = D / 8, PPW = 64 / L, U = 4;  // pages per load, loads in flight
  const int lane = threadIdx.x & 63, sub = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SelectRow row = rows.r[row_index(rows.r, &SelectRow::item0, (int)blockIdx.x)];
  const int chunks = (row.stride + kScorePages - 1) / kScorePages;
  const int x = (int)blockIdx.x - row.item0;
  const int chunk = x % chunks, h = x / chunks % a.hkv, j = x / chunks / a.hkv;
  const int n_pages = (row.start + j) / a.block + 1;  // of this token
  const int p0 = chunk * kScorePages, p1 = min(n_pages, p0 + kScorePages);
  if (p0 >= p1) return;
  const int64_t t = (int64_t)row.tok0 + j;
  double qd[G][8];
#pragma unroll
  for (int e = 0; e < G; ++e) {
    const uint4 v = cpattn::ld_global16(q + (t * a.hq + h * G + e) * D + sub * 8);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) qd[e][i] = (double)(i & 1 ? bf16hi(w[i / 2]) : bf16lo(w[i / 2]));
  }
  const int32_t* bt_row = bt + (int64_t)row.req * a.mbr;
  uint64_t* dst = scores + row.score0 + ((int64_t)j * a.hkv + h) * row.stride;
  const int group = lane / L;
  for (int b = p0 + wave * PPW * U; b < p1; b += kWaves * PPW * U) {
    uint4 lo[U], hi[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int page = min(b + u * PPW + group, p1 - 1);  // past the last page that one again
      const int blk = bt_row[page];
      there[u] = blk >= 0 && blk < a.num_blocks;
      const uint4* src = bounds + ((int64_t)(there[u] ? blk : 0) * a.hkv + h) * 2 * L + sub;
      lo[u] = cpattn::ld_global16(src);
      hi[u] = cpattn::ld_global16(src + L);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t lw[4] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w};
      const uint32_t hw[4] = {hi[u].x, hi[u].y, hi[u].z, hi[u].w};
      double s[G];
#pragma unroll
      for (int e = 0; e < G; ++e) s[e] = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double l = i & 1 ? bf16hi(lw[i / 2]) : bf16lo(lw[i / 2]);
        const double m = i & 1 ? bf16hi(hw[i / 2]) : bf16lo(hw[i / 2]);
        const double both = l + m, width = m - l;
#pragma unroll
        for (int e = 0; e < G; ++e)
          s[e] = __builtin_fma(fabs(qd[e][i]), width, __builtin_fma(qd[e][i], both, s[e]));
      }
      // sums over the L lanes, then the largest of the heads
      constexpr int N1 = L == 16 ? (G > 1 ? G / 2 : 1) : G, N2 = N1 > 1 ? N1 / 2 : 1,
                    N3 = N2 > 1 ? N2 / 2 : 1;
      if constexpr (L == 16) sum_step<8, G>(s, lane);
      sum_step<4, N1>(s, lane);
      sum_step<2, N2>(s, lane);
      sum_step<1, N3>(s, lane);
      static_assert(N3 <= 2, "one head's sum is left");
      uint64_t k = key_of(s[0]);
      if constexpr (N3 > 1) k = max_step<1>(k);
      if constexpr (N2 > 1) k = max_step<2>(k);
      if constexpr (N1 > 1) k = max_step<4>(k);
      if constexpr (L == 16 && G > 1) k = max_step<8>(k);
      const int page = b + u * PPW + group;
      if (sub == 0 && page < p1) dst[page] = there[u] ? k : 0;
    }
  }
}

// Exclusive sum of x over the workgroup's threads; `total` gets the whole.
__device__ __forceinline__ int scan(int x, int* s_wave, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(sum, d, 64);
    if (lane >= d) sum += o;
  }
  __syncthreads();  // s_wave's last use
  if (lane == 63) s_wave[wave] = sum;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    if (w < wave) before += s_wave[w];
    all += s_wave[w];
  }
  *total = all;
  return before + sum - x;
}

// The choice: one workgroup per (token, kv head).  The n_pages-th largest key is
// found eight bits at a time, from a histogram of the keys that agree with the
// bits known so far; then the pages are written in order, those above it and
// as many equal ones as there is room for, the lower first.
template <class Rows>
__global__ __launch_bounds__(kThreads) void choose_kernel(const Rows rows, const SelectArgs a,
                                                          const uint64_t* __restrict__ scores) {
  __shared__ int s_hist[256];
  __shared__ int s_wave[kWaves];
  __shared__ int s_digit, s_left;
  const SelectRow row = rows.r[row_index(rows.r, &SelectRow::item0, (int)blockIdx.x)];
  const int x = (int)blockIdx.x - row.item0, h = x % a.hkv, j = x / a.hkv;
  const int64_t t = (int64_t)row.tok0 + j;
  int32_t* dst = a.pages + (t * a.hkv + h) * a.n_pages;
  const int n = (row.start + j) / a.block + 1, P = a.n_pages, tid = threadIdx.x;
  if (n <= P) {  // all of them
    for (int i = tid; i < P; i += kThreads) dst[i] = i < n ? i : -1;
    return;
  }
  const uint64_t* src = scores + row.score0 + ((int64_t)j * a.hkv + h) * row.stride;
  const auto key = [&](int i) { return i < a.n_first || i >= n - a.n_last ? kForcedKey : src[i]; };
  uint64_t known = 0;  // the bits of the threshold found so far
  int left = P;        // of the keys that agree with them, how many are selected
  for (int shift = 56; shift >= 0; shift -= 8) {
    s_hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint64_t k = key(i);
      if (shift == 56 || k >> (shift + 8) == known >> (shift + 8))
        atomicAdd(&s_hist[(int)(k >> shift) & 255], 1);
    }
    __syncthreads();
    // thread d: the keys with a larger digit
    int total;
    const int mine = s_hist[255 - tid];
    const int above = scan(mine, s_wave, &total);
    if (above < left && above + mine >= left) s_digit = 255 - tid, s_left = left - above;
    __syncthreads();
    known |= (uint64_t)s_digit << shift;
    left = s_left;
  }
  // in order, kThreads at a time
  int out = 0;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    const int i = i0 + tid;
    const uint64_t k = i < n ? key(i) : 0;
    const bool equal = i < n && k == known;
    int equals, chosen;
    const int rank = scan(equal ? 1 : 0, s_wave, &equals);
    const bool take = i < n && (k > known || (equal && rank < left));
    const int at = scan(take ? 1 : 0, s_wave, &chosen);
    if (take) dst[out + at] = i;
    out += chosen;
    left -= min(left, equals);
  }
}

template <int D, int G>
hipError_t launch_score_t(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                          hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL((score_kernel<D, G>), dim3(items), dim3(kThreads), 0, s, r, a, a.q,
                       (const uint4*)a.bounds, a.bt, a.scores);
  });
}

}  // namespace

hipError_t launch_score(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                        hipStream_t s) {
  switch (a.hq / a.hkv) {
    case 1: return (d == 128 ? launch_score_t<128, 1> : launch_score_t<64, 1>)(a, rows, n_rows, items, s);
    case 2: return (d == 128 ? launch_score_t<128, 2> : launch_score_t<64, 2>)(a, rows, n_rows, items, s);
    case 4: return (d == 128 ? launch_score_t<128, 4> : launch_score_t<64, 4>)(a, rows, n_rows, items, s);
    case 8: return (d == 128 ? launch_score_t<128, 8> : launch_score_t<64, 8>)(a, rows, n_rows, items, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_choose(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL(choose_kernel, dim3(items), dim3(kThreads), 0, s, r, a, a.scores);
  });
}

}  // namespace cpcache
