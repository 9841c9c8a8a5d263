// Selection of pages by the bounds of their keys (include/cp_cache.h).
//
// The score of a page is the largest product that a key within its bounds can
// have with one of a group's q heads.  Which pages are selected hangs on the
// order of the scores, so they are fp64: products of bf16 are exact in it and
// their sums are, for all but extreme values, too, whatever their order.
#include <type_traits>

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

template <int Ctrl>
__device__ __forceinline__ uint64_t dpp64(uint64_t x) {
  const float lo = cpattn::dpp<Ctrl>(__uint_as_float((uint32_t)x));
  const float hi = cpattn::dpp<Ctrl>(__uint_as_float((uint32_t)(x >> 32)));
  return (uint64_t)__float_as_uint(lo) | (uint64_t)__float_as_uint(hi) << 32;
}

// The value of the lane whose index differs in bit Bit alone (1, 2, 4 or 8).
template <int Bit>
__device__ __forceinline__ uint64_t partner64(uint64_t x) {
  if constexpr (Bit == 4) return dpp64<0x1B>(dpp64<cpattn::kMirror8>(x));  // 7 - i, then i ^ 3
  else return dpp64<Bit == 1 ? cpattn::kXor1 : Bit == 2 ? cpattn::kXor2 : cpattn::kXor8>(x);
}
// The same but for Bit 4, where the bits below differ, too.
template <int Bit>
__device__ __forceinline__ uint64_t mirror64(uint64_t x) {
  if constexpr (Bit == 4) return dpp64<cpattn::kMirror8>(x);
  else return partner64<Bit>(x);
}

// One step of a sum over lanes that differ in `Bit`: of N sums a lane keeps one
// half, by its side, and gives away the other; the last one both sides keep.
template <int Bit, int N>
__device__ __forceinline__ void sum_step(double* u, int lane) {
  const auto add = [](double keep, double give) {
    return keep + __longlong_as_double(
                      (long long)mirror64<Bit>((uint64_t)__double_as_longlong(give)));
  };
  if constexpr (N > 1) {
    const bool up = lane & Bit;
#pragma unroll
    for (int e = 0; e < N / 2; ++e)
      u[e] = add(up ? u[e + N / 2] : u[e], up ? u[e] : u[e + N / 2]);
  } else {
    u[0] = add(u[0], u[0]);
  }
}

// Scores of pages [p0, p1) of kv head h of token t, by the NW waves of a workgroup:
// store(page, key).  A wave takes 64 / L pages at a time, L = D / 8 lanes a page with
// 8 features each.  With lo + hi and hi - lo of a feature, whichever is the larger,
//     2 max(q lo, q hi) = q (lo + hi) + |q| |hi - lo|:
// two fp64 multiply-adds per head and feature.  Sums over a page's lanes are split
// by head first, then by the U pages that the lanes have in hand.  At 4 heads a
// group that is some 170 vector operations per 2 KB of bounds.  (On the fp64 matrix
// instructions, 4x4x4 in four blocks, the scores of 32 requests of ~34,000 keys took
// 78 us on 32/8 heads and 189 on 64/8, here 53 and 76.)  Those 53 us move 246 MB,
// 4.6 TB/s: the loads and the fp64 units take turns at being the slower.
template <int D, int G, int NW, class Store>
__device__ __forceinline__ void score_pages(const SelectArgs& a, int64_t t, int h,
                                            const int32_t* __restrict__ bt_row, int p0, int p1,
                                            const uint16_t* __restrict__ q,
                                            const uint4* __restrict__ bounds, Store&& store) {
  constexpr int L = D / 8, PPW = 64 / L, U = 4;  // pages per load, loads in flight
  // heads per lane behind the steps over lane bits 4 and 8
  constexpr int H4 = G > 1 ? G / 2 : 1, H = L == 16 && H4 > 1 ? H4 / 2 : H4;
  const int lane = threadIdx.x & 63, sub = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = lane / L;
  constexpr int STEP = NW * PPW * U;
  const int begin = p0 + wave * PPW * U;
  if (begin >= p1) return;  // whole wave
  // past the last page that one again
  const auto entry = [&](int b, int u) { return bt_row[min(b + u * PPW + group, p1 - 1)]; };
  const auto there = [&](int blk) { return blk >= 0 && blk < a.num_blocks; };
  int32_t blk[U], blk_next[U];
  uint4 lo[U], hi[U];
  const auto load = [&](int u, int at) {
    const uint4* src = bounds + ((int64_t)(there(at) ? at : 0) * a.hkv + h) * 2 * L + sub;
    lo[u] = cpattn::ld_global16_nt(src);
    hi[u] = cpattn::ld_global16_nt(src + L);
  };
#pragma unroll
  for (int u = 0; u < U; ++u) blk[u] = entry(begin, u);
  double qd[G][8];
#pragma unroll
  for (int e = 0; e < G; ++e) {
    const uint4 v = cpattn::ld_global16(q + (t * a.hq + h * G + e) * D + sub * 8);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) qd[e][i] = (double)(i & 1 ? bf16hi(w[i / 2]) : bf16lo(w[i / 2]));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, blk[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) blk_next[u] = entry(begin + STEP, u);
  for (int b = begin; b < p1; b += STEP) {
    double sum[U * H];
    uint32_t found = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t lw[4] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w};
      const uint32_t hw[4] = {hi[u].x, hi[u].y, hi[u].z, hi[u].w};
      // the next pages' bounds are on their way while these are in use
      found |= there(blk[u]) ? 1u << u : 0u;
      blk[u] = blk_next[u];
      load(u, blk[u]);
      blk_next[u] = entry(b + 2 * STEP, u);
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
          s[e] = __builtin_fma(fabs(qd[e][i]), fabs(width), __builtin_fma(qd[e][i], both, s[e]));
      }
      sum_step<4, G>(s, lane);
      if constexpr (L == 16) sum_step<8, H4>(s, lane);
#pragma unroll
      for (int e = 0; e < H; ++e) sum[u * H + e] = s[e];
    }
    static_assert(U == 4, "two lane bits");
    sum_step<2, U * H>(sum, lane);
    sum_step<1, U / 2 * H>(sum, lane);
    // lane bits 1 and 0 name the page, bits 8 and 4 the heads
    uint64_t k = key_of(sum[0]);
#pragma unroll
    for (int e = 1; e < H; ++e) k = max(k, key_of(sum[e]));
    if constexpr (G > 1) k = max(k, partner64<4>(k));
    if constexpr (L == 16 && H4 > 1) k = max(k, partner64<8>(k));
    const int u = lane & 3, page = b + u * PPW + group;
    if (sub < U && page < p1) store(page, found >> u & 1 ? k : 0);
  }
}

// A workgroup of the scores takes a.chunk pages of one (token, kv head).
template <int D, int G, class Rows>
__global__ __launch_bounds__(kThreads, G <= 4 ? 4 : 2) void score_kernel(
    const Rows rows, const SelectArgs a, const uint16_t* __restrict__ q,
    const uint4* __restrict__ bounds, const int32_t* __restrict__ bt,
    uint64_t* __restrict__ scores) {
  const SelectRow row = rows.r[row_index(rows.r, &SelectRow::item0, (int)blockIdx.x)];
  const int chunks = (row.stride + a.chunk - 1) / a.chunk;
  const int x = (int)blockIdx.x - row.item0;
  const int chunk = x % chunks, h = x / chunks % a.hkv, j = x / chunks / a.hkv;
  const int p0 = chunk * a.chunk, p1 = min((row.start + j) / a.block + 1, p0 + a.chunk);
  if (p0 >= p1) return;
  uint64_t* dst = scores + row.score0 + ((int64_t)j * a.hkv + h) * row.stride;
  score_pages<D, G, kWaves>(a, (int64_t)row.tok0 + j, h, bt + (int64_t)row.req * a.mbr, p0, p1, q,
                            bounds, [&](int page, uint64_t key) { dst[page] = key; });
}

// Inclusive sum of x over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

// The largest of x over groups of 16 lanes, and over the wave.
__device__ __forceinline__ uint64_t max16(uint64_t x) {
  x = max(x, partner64<1>(x));
  x = max(x, partner64<2>(x));
  x = max(x, mirror64<4>(x));
  return max(x, partner64<8>(x));
}
__device__ __forceinline__ uint64_t max64(uint64_t x) {
  x = max16(x);
  x = max(x, (uint64_t)__shfl_xor((unsigned long long)x, 16, 64));
  return max(x, (uint64_t)__shfl_xor((unsigned long long)x, 32, 64));
}

// A (token, kv head) that selects: item blockIdx.x of the launch.
struct Choice {
  int n;  // pages to choose from
  int64_t t;
  int h, req;
  int64_t score0;  // the first of its scores
};

template <class Rows>
__device__ __forceinline__ Choice choice_of(const Rows& rows, const SelectArgs& a) {
  const SelectRow row = rows.r[row_index(rows.r, &SelectRow::item0, (int)blockIdx.x)];
  const int x = (int)blockIdx.x - row.item0, h = x % a.hkv, j = x / a.hkv;
  return Choice{(row.start + j) / a.block + 1, (int64_t)row.tok0 + j, h, row.req,
                row.score0 + ((int64_t)j * a.hkv + h) * row.stride};
}

// The choice of a.n_pages of n > a.n_pages pages, by a workgroup of NT threads that
// holds up to NT NU keys, src(page), in registers.  The fixed pages aside, the
// place of the threshold is found eight bits at a time from the highest one in
// which the keys differ, by a histogram of the keys that agree with the bits known
// so far.  Once few keys are left, or all of them are selected, each counts those
// before it.  The selected pages are written in order, by the ballots of the waves.
// Bound by its barriers, some three a digit: 8.7 us for 128 of ~2,100 pages, 256 (token, kv
// head)s; 5.1 for 32 of 256 pages, 8 of them.
template <int NT, int NU, class Src>
__device__ __forceinline__ void choose_pages(const SelectArgs& a, int n, Src&& src, int32_t* dst) {
  constexpr int NW = NT / 64, SH = 8, kFew = NT / SH, NC = NU * NW, CPL = NC > 64 ? NC / 64 : 1;
  static_assert(NW <= 16 && NT % SH == 0 && (NC <= 64 || NC == 64 * CPL), "geometry");
  __shared__ __align__(16) int s_hist[2][256];
  __shared__ int s_count[2][CPL * 64];
  __shared__ uint64_t s_max[16], s_not_min[16], s_key[kFew];
  __shared__ int s_page[kFew], s_digit, s_left, s_in, s_few;
  __shared__ unsigned long long s_take[NC];
  const int P = a.n_pages, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // n > P >= fixed pages: those are apart
  const int first = a.n_first, last = n - a.n_last;  // chosen from: [first, last)
  uint64_t key[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int i = u * NT + tid;
    key[u] = i >= first && i < last ? src(i) : 0;
  }
  for (int x = tid; x < 512; x += NT) s_hist[x >> 8][x & 255] = 0;
  if (tid < 2 * CPL * 64) s_count[0][tid] = 0;  // (NT >= 2 CPL 64)
  static_assert(NT >= 2 * CPL * 64 && NT >= NC, "one word a thread");
  if (tid < NC) s_take[tid] = 0;
  if (tid == 0) s_few = 0;
  uint64_t most = 0, not_least = 0;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int i = u * NT + tid;
    if (i >= first && i < last) most = max(most, key[u]), not_least = max(not_least, ~key[u]);
  }
  most = max64(most), not_least = max64(not_least);
  if (lane == 0) s_max[wave] = most, s_not_min[wave] = not_least;
  __syncthreads();
  most = max16(s_max[min(lane & 15, NW - 1)]);
  const uint64_t least = ~max16(s_not_min[min(lane & 15, NW - 1)]);
  int left = P - a.n_first - a.n_last;  // still to be chosen, of `in` keys that agree with
  int in = last - first;                // `known` in the bits from `shift` on
  int shift = 64 - __clzll((long long)(most ^ least));  // (of equal ones: 0)
  uint64_t known = shift < 64 ? most >> shift : 0;
  for (int pass = 0; in > kFew && in > left && left > 0 && shift > 0; pass ^= 1) {
    const int low = max(0, shift - 8), bits = shift - low;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = u * NT + tid;
      if (i >= first && i < last && (shift >= 64 || key[u] >> shift == known))
        atomicAdd(&s_hist[pass][(int)(key[u] >> low) & ((1 << bits) - 1)], 1);
    }
    __syncthreads();
    if (wave == 0) {  // lane l: digits 255 - 4 l and the three below
      const int4 d = *reinterpret_cast<const int4*>(&s_hist[pass][252 - 4 * lane]);
      const int upto = wave_scan(d.x + d.y + d.z + d.w);
      const int c3 = upto - d.x - d.y - d.z - d.w;  // above digit 255 - 4 l
      const int c2 = c3 + d.w, c1 = c2 + d.z, c0 = c1 + d.y;
      if (c3 < left && upto >= left) {
        const int x = c2 >= left ? 3 : c1 >= left ? 2 : c0 >= left ? 1 : 0;
        s_digit = 252 - 4 * lane + x;
        s_left = left - (x == 3 ? c3 : x == 2 ? c2 : x == 1 ? c1 : c0);
        s_in = x == 3 ? d.w : x == 2 ? d.z : x == 1 ? d.y : d.x;
      }
    } else {
      for (int x = tid - 64; x < 256; x += NT - 64) s_hist[pass ^ 1][x] = 0;
    }
    __syncthreads();
    known = (shift < 64 ? known << bits : 0) | (uint64_t)s_digit;
    left = s_left, in = s_in, shift = low;
  }
  // above the agreeing keys: chosen; of those, all, none, or the `left` first by
  // (key, page)
  uint32_t chosen = 0, agree = 0;  // a bit per u
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int i = u * NT + tid;
    const uint64_t top = shift < 64 ? key[u] >> shift : 0;
    const bool fixed = i < first || (i >= last && i < n);
    if (fixed || (i < last && top > known)) chosen |= 1u << u;
    else if (i < last && top == known) agree |= 1u << u;
  }
  // word x of a wave's counts (u, wave) of the keys before
  const auto count = [&](uint32_t bits, int buffer, int (&before)[CPL]) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const uint64_t b = __builtin_amdgcn_ballot_w64(bits >> u & 1);
      if (lane == 0) s_count[buffer][u * NW + wave] = __popcll(b);
    }
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int x = 0; x < CPL; ++x) {
      before[x] = sum;
      sum += s_count[buffer][CPL * lane + x];
    }
    const int lanes_before = wave_scan(sum) - sum;
#pragma unroll
    for (int x = 0; x < CPL; ++x) before[x] += lanes_before;
  };
  const auto position = [&](uint32_t bits, int u, const int (&before)[CPL]) {
    const uint64_t b = __builtin_amdgcn_ballot_w64(bits >> u & 1);
    const int word = u * NW + wave;
    int at = 0;
#pragma unroll
    for (int x = 0; x < CPL; ++x)
      if (word % CPL == x) at = __builtin_amdgcn_readlane(before[x], word / CPL);
    return at + __popcll(b & ((1ull << lane) - 1));
  };
  if (in <= left) {
    chosen |= agree;
  } else if (left > 0 && in <= kFew) {
#pragma unroll
    for (int u = 0; u < NU; ++u)
      if (agree >> u & 1) {
        const int at = atomicAdd(&s_few, 1);
        s_key[at] = key[u], s_page[at] = u * NT + tid;
      }
    __syncthreads();
    // SH threads count the keys before one (whatever their order here); two of them,
    // and up to 128 keys, took 5 us of a workgroup of four waves
    const int e0 = tid % SH, x = min(tid / SH, in - 1);
    const uint64_t k = s_key[x];
    const int page = s_page[x];
    int before = 0;
#pragma unroll 4
    for (int e = e0; e < in; e += SH)
      before += s_key[e] > k || (s_key[e] == k && s_page[e] < page);
#pragma unroll
    for (int m = 1; m < SH; m <<= 1) before += __shfl_xor(before, m, 64);
    if (e0 == 0 && tid / SH < in && before < left)
      atomicOr(&s_take[page >> 6], 1ull << (page & 63));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < NU; ++u) chosen |= (uint32_t)(s_take[u * NW + wave] >> lane & 1) << u;
  } else if (left > 0) {  // more equal keys: the first `left`
    int before[CPL];
    count(agree, 1, before);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int at = position(agree, u, before);
      if ((agree >> u & 1) && at < left) chosen |= 1u << u;
    }
  }
  int before[CPL];
  count(chosen, 0, before);
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int at = position(chosen, u, before);
    if (chosen >> u & 1) dst[at] = u * NT + tid;
  }
}

// All of n <= a.n_pages pages.
__device__ __forceinline__ void take_all(const SelectArgs& a, int n, int32_t* dst) {
  for (int i = threadIdx.x; i < a.n_pages; i += blockDim.x) dst[i] = i < n ? i : -1;
}

template <int NT, int NU, class Rows>
__global__ __launch_bounds__(NT) void choose_kernel(const Rows rows, const SelectArgs a,
                                                    const uint64_t* __restrict__ scores) {
  const Choice c = choice_of(rows, a);
  int32_t* dst = a.pages + (c.t * a.hkv + c.h) * a.n_pages;
  if (c.n <= a.n_pages) return take_all(a, c.n, dst);
  const uint64_t* src = scores + c.score0;
  choose_pages<NT, NU>(a, c.n, [&](int i) { return src[i]; }, dst);
}

// Scores and choice in one, for up to NP pages a token.
template <int G>
constexpr int kOneThreads = G <= 4 ? 1024 : 512;  // (128 and 256 registers a lane)
template <int D, int G, int NT, int NP, class Rows>
__global__ __launch_bounds__(NT, G <= 4 ? 4 : 2) void select_kernel(
    const Rows rows, const SelectArgs a, const uint16_t* __restrict__ q,
    const uint4* __restrict__ bounds, const int32_t* __restrict__ bt) {
  __shared__ uint64_t s_score[NP];
  const Choice c = choice_of(rows, a);
  int32_t* dst = a.pages + (c.t * a.hkv + c.h) * a.n_pages;
  if (c.n <= a.n_pages) return take_all(a, c.n, dst);
  score_pages<D, G, NT / 64>(a, c.t, c.h, bt + (int64_t)c.req * a.mbr, 0, c.n, q, bounds,
                             [&](int page, uint64_t key) { s_score[page] = key; });
  __syncthreads();
  choose_pages<NT, NP / NT>(a, c.n, [&](int i) { return s_score[i]; }, dst);
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

// The same for more keys than a workgroup holds, which are read again in each pass.
// Bound by the latency of nine passes by four waves: 179 us for 128 of 16,385 pages, 8
// (token, kv head)s (of 16,384, held in registers, 14.5; their scores 19), 268 for 256 of
// them (23; 390), and twice that of 32,768 pages.
template <class Rows>
__global__ __launch_bounds__(kThreads) void choose_long_kernel(const Rows rows, const SelectArgs a,
                                                               const uint64_t* __restrict__ scores) {
  __shared__ int s_hist[256];
  __shared__ int s_wave[kWaves];
  __shared__ int s_digit, s_left;
  const Choice c = choice_of(rows, a);
  int32_t* dst = a.pages + (c.t * a.hkv + c.h) * a.n_pages;
  if (c.n <= a.n_pages) return take_all(a, c.n, dst);
  const uint64_t* src = scores + c.score0;
  const int n = c.n, P = a.n_pages, tid = threadIdx.x;
  const auto key = [&](int i) {
    return i < a.n_first || i >= n - a.n_last ? kForcedKey : src[i];
  };
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

template <int X>
using N = std::integral_constant<int, X>;

template <int D, int G>
hipError_t launch_score_t(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                          One one, hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    const auto both = [&](auto threads, auto pages) {
      constexpr int NT = decltype(threads)::value, NP = decltype(pages)::value;
      hipLaunchKernelGGL((select_kernel<D, G, NT, NP>), dim3(items), dim3(NT), 0, s, r, a, a.q,
                         (const uint4*)a.bounds, a.bt);
    };
    switch (one) {
      case One::kFour256: return both(N<kThreads>(), N<256>());
      case One::kFour1024: return both(N<kThreads>(), N<1024>());
      case One::kAll1024: return both(N<kOneThreads<G>>(), N<1024>());
      case One::kNo: break;
    }
    hipLaunchKernelGGL((score_kernel<D, G>), dim3(items), dim3(kThreads), 0, s, r, a, a.q,
                       (const uint4*)a.bounds, a.bt, a.scores);
  });
}

hipError_t launch_score_g(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                          One one, hipStream_t s) {
  const auto f = [&](auto g) {
    constexpr int G = decltype(g)::value;
    return d == 128 ? launch_score_t<128, G>(a, rows, n_rows, items, one, s)
                    : launch_score_t<64, G>(a, rows, n_rows, items, one, s);
  };
  switch (a.hq / a.hkv) {
    case 1: return f(N<1>());
    case 2: return f(N<2>());
    case 4: return f(N<4>());
    case 8: return f(N<8>());
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_score(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                        hipStream_t s) {
  return launch_score_g(d, a, rows, n_rows, items, One::kNo, s);
}

hipError_t launch_select(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         One one, hipStream_t s) {
  return launch_score_g(d, a, rows, n_rows, items, one, s);
}

hipError_t launch_choose(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         int most, hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    const auto held = [&](auto threads, auto keys) {
      constexpr int NT = decltype(threads)::value, NU = decltype(keys)::value;
      hipLaunchKernelGGL((choose_kernel<NT, NU>), dim3(items), dim3(NT), 0, s, r, a, a.scores);
    };
    if (most <= kFewPages) held(N<choose_threads(kFewPages)>(), N<4>());
    else if (most <= kSomePages) held(N<choose_threads(kSomePages)>(), N<4>());
    else if (most <= kManyPages) held(N<choose_threads(kManyPages)>(), N<16>());
    else
      hipLaunchKernelGGL(choose_long_kernel, dim3(items), dim3(kThreads), 0, s, r, a, a.scores);
  });
}

}  // namespace cpcache
