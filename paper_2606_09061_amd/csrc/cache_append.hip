// Rotation and append in one launch, and the bounds of the written pages
// (include/cp_cache.h).
#include "cache_device.hpp"

namespace cpcache {

using cpattn::bf16hi;
using cpattn::bf16lo;
using cpattn::to_bf16;
using cpattn::u32x4_t;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ uint32_t pack(float a, float b) {
  return (uint32_t)to_bf16(a) | ((uint32_t)to_bf16(b) << 16);
}

__device__ __forceinline__ float sumsq8(const uint4& a) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s += bf16lo(w[i]) * bf16lo(w[i]) + bf16hi(w[i]) * bf16hi(w[i]);
  return s;
}

// Lanes of 8 x 8 tiles of V that a (page, kv head) needs, and kv heads per wave.
template <int D, int B>
struct VGeom {
  static constexpr int NTS = B / 8, NFG = D / 8, LANES = NTS * NFG, HEADS = 64 / LANES;
  static_assert(LANES <= 64, "a page's tiles fit a wave");
};

// Workgroups [0, rope_blocks): one wave per (token, part of its q and k heads).
// A head is D / 8 consecutive lanes of 8 elements; lane j < D / 16 of a head
// holds elements of the first half and lane j + D / 16 their rotation partners,
// and the two swap their raw words with one cross-lane exchange.  The rotation
// is the same for all heads of a token: its sines and cosines, formed in turns
// and reduced in fp64 (some 6 fp64 operations per element), are made once per
// wave and kept for all heads that it takes.  The arithmetic is
// cpl_qkv_rope's, operation by operation, for the same bits.
//
// The others: one wave per item of V, a page's new tokens for VGeom::HEADS kv
// heads.  A page holds V feature-major: a lane takes 8 slots x 8 features
// through registers and writes runs of 8 slots (16 bytes) where all are new.
//
// Bound by HBM: 2,048 tokens on 64/8 heads of 128 take 19.0 us for 84 MB, 4.4 TB/s
// (a large copy: 4.9); 64 decode rows on 32/8 5.7 us and one row 4.2, a launch's
// latency.
template <int D, int B, class Rows>
__global__ __launch_bounds__(kThreads) void append_kernel(
    const Rows rows, const AppendArgs a, int tokens, int parts, int rope_blocks, int v_items,
    const uint4* __restrict__ qkv, const uint4* __restrict__ qw, const uint4* __restrict__ kw,
    const int32_t* __restrict__ positions, const int32_t* __restrict__ bt, uint4* __restrict__ q,
    uint16_t* __restrict__ k_cache, uint16_t* __restrict__ v_cache) {
  constexpr int L = D / 8, HPW = 64 / L, HALF = L / 2;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hq = a.hq, hkv = a.hkv, nh = hq + 2 * hkv;
  if ((int)blockIdx.x < rope_blocks) {
    const int64_t w = (int64_t)blockIdx.x * kWaves + wave;
    if (w >= (int64_t)tokens * parts) return;
    const int x = (int)(w / parts), part = (int)(w % parts);
    const AppendRow row = rows.r[row_index(rows.r, &AppendRow::first, x)];
    const int64_t t = (int64_t)row.tok0 + x - row.first;
    const int slot = row.start + x - row.first;
    const int64_t blk = bt[(int64_t)row.req * a.mbr + slot / B];
    const bool placed = blk >= 0 && blk < a.num_blocks;
    const int sub = lane % L, mlo = sub % HALF;
    // frequency of element e in turns per position:
    // theta^(-2 (8 (sub mod D/16) + e) / D) / (2 pi) = step8^(sub mod D/16) * step^e / (2 pi)
    double f = 0.15915494309189533576888376337251, p = a.step8;
#pragma unroll
    for (int bit = 0; bit < 3; ++bit) {
      if (mlo & (1 << bit)) f *= p;
      p *= p;
    }
    const double pos = (double)(positions ? positions[t] : slot);
    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = pos * f;
      f *= a.step;
      const float r = (float)(turns - rint(turns));
      sn[e] = __builtin_amdgcn_sinf(r), cs[e] = __builtin_amdgcn_cosf(r);
    }
    const float sgn = sub < HALF ? -1.f : 1.f;
    const int groups = (hq + hkv + HPW - 1) / HPW;
    const uint4 own[2] = {qw[sub], kw[sub]}, partner[2] = {qw[sub ^ HALF], kw[sub ^ HALF]};
    for (int g = part; g < groups; g += parts) {
      const int hh = g * HPW + lane / L;
      const bool live = hh < hq + hkv;
      const uint4 x4 = live ? qkv[((size_t)t * nh + hh) * L + sub] : make_uint4(0, 0, 0, 0);
      uint4 y4;  // the partner lane's raw words
      y4.x = __shfl_xor(x4.x, HALF, 64);
      y4.y = __shfl_xor(x4.y, HALF, 64);
      y4.z = __shfl_xor(x4.z, HALF, 64);
      y4.w = __shfl_xor(x4.w, HALF, 64);
      float ss = sumsq8(x4);
#pragma unroll
      for (int m = 1; m < L; m <<= 1) ss += __shfl_xor(ss, m, 64);
      const float scale = 1.0f / sqrtf(ss / (float)D + a.eps);
      const bool is_q = hh < hq;
      const uint4 wo = is_q ? own[0] : own[1], wp = is_q ? partner[0] : partner[1];
      const uint32_t aw[4] = {x4.x, x4.y, x4.z, x4.w}, bw[4] = {y4.x, y4.y, y4.z, y4.w};
      const uint32_t wow[4] = {wo.x, wo.y, wo.z, wo.w}, wpw[4] = {wp.x, wp.y, wp.z, wp.w};
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float r2[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float xo = (h ? bf16hi(aw[i]) : bf16lo(aw[i])) * scale *
                           (h ? bf16hi(wow[i]) : bf16lo(wow[i]));
          const float xp = (h ? bf16hi(bw[i]) : bf16lo(bw[i])) * scale *
                           (h ? bf16hi(wpw[i]) : bf16lo(wpw[i]));
          r2[h] = xo * cs[2 * i + h] + sgn * (xp * sn[2 * i + h]);
        }
        o[i] = pack(r2[0], r2[1]);
      }
      const uint4 out = make_uint4(o[0], o[1], o[2], o[3]);
      if (!live) continue;
      if (is_q)
        q[((size_t)t * hq + hh) * L + sub] = out;
      else if (placed)
        *reinterpret_cast<uint4*>(k_cache + ((blk * hkv + hh - hq) * B + slot % B) * D + sub * 8) =
            out;
    }
    return;
  }

  using V = VGeom<D, B>;
  const int64_t item = (int64_t)((int)blockIdx.x - rope_blocks) * kWaves + wave;
  if (item >= v_items) return;
  const AppendRow row = rows.r[row_index(rows.r, &AppendRow::item0, (int)item)];
  const int per = (hkv + V::HEADS - 1) / V::HEADS;  // items per page
  const int y = (int)item - row.item0, lb = row.start / B + y / per;
  const int h = y % per * V::HEADS + lane / V::LANES;
  const int64_t blk = bt[(int64_t)row.req * a.mbr + lb];
  const int end = row.start + row.n;  // the piece's last token + 1
  const int slot0 = max(row.start, lb * B) - lb * B, slot1 = min(end, (lb + 1) * B) - lb * B;
  const int ts = lane % V::LANES / V::NFG, fg = lane % V::NFG;
  const int s_lo = max(8 * ts, slot0), s_hi = min(8 * ts + 8, slot1);
  if (h >= hkv || s_lo >= s_hi || blk < 0 || blk >= a.num_blocks) return;
  u32x4_t w[8];  // w[e]: token in slot 8 ts + e, features 8 fg .. 8 fg + 7
#pragma unroll
  for (int e = 0; e < 8; ++e) {  // slots outside the span re-read one inside it
    const int slot = min(max(8 * ts + e, s_lo), s_hi - 1);
    const int64_t t = (int64_t)row.tok0 + lb * B + slot - row.start;
    w[e] = reinterpret_cast<const u32x4_t*>(qkv)[((size_t)t * nh + hq + hkv + h) * L + fg];
  }
  uint16_t* dst = v_cache + ((blk * hkv + h) * D + fg * 8) * B + 8 * ts;
  const bool whole = s_lo == 8 * ts && s_hi == 8 * ts + 8;
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    uint32_t v16[8];  // feature 8 fg + f of the 8 slots
#pragma unroll
    for (int e = 0; e < 8; ++e) v16[e] = (w[e][f / 2] >> (16 * (f % 2))) & 0xffffu;
    if (whole) {
      u32x4_t o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = v16[2 * i] | (v16[2 * i + 1] << 16);
      *reinterpret_cast<u32x4_t*>(dst + f * B) = o;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * ts + e >= s_lo && 8 * ts + e < s_hi) dst[f * B + e] = (uint16_t)v16[e];
    }
  }
}

// One wave per (page, kv head): lane l reads 16-byte piece l % (D / 8) of every
// 64 / (D / 8)-th key, keeps its features' extremes and shares them with the
// lanes of the same piece.  Bound by the stream of K: 32,768 tokens, 8 kv heads of
// 128, pages of 16, take 17.1 us for 76 MB, 4.4 TB/s; 64 rows' last pages 4.1.  Two or
// four kv heads a wave, which keep more loads on their way, took 17.5 and 19.4.
template <int D, int B, class Rows>
__global__ __launch_bounds__(kThreads) void bounds_kernel(const Rows rows, const BoundsArgs a,
                                                          int items,
                                                          const uint16_t* __restrict__ k_cache,
                                                          const int32_t* __restrict__ bt,
                                                          uint4* __restrict__ bounds) {
  constexpr int L = D / 8, KPL = 64 / L, NL = B / KPL;  // lanes per key, keys per load, loads
  constexpr float kMax = 3.3895313892515355e38f;        // the largest finite bf16
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
  if (item >= items) return;
  const int x = (int)(item / a.hkv), h = (int)(item % a.hkv);
  const BoundsRow row = rows.r[row_index(rows.r, &BoundsRow::item0, x)];
  const int lb = row.page0 + x - row.item0, held = min(B, row.ctx - lb * B);
  const int64_t blk = bt[(int64_t)row.req * a.mbr + lb];
  if (blk < 0 || blk >= a.num_blocks) return;
  const uint16_t* base = k_cache + (blk * a.hkv + h) * B * D + lane % L * 8;
  uint4 k[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)  // past the last key that one again
    k[i] = cpattn::ld_global16_nt(base + min(i * KPL + lane / L, held - 1) * D);
  float lo[8], hi[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) lo[e] = INFINITY, hi[e] = -INFINITY;
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const uint32_t w[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = e & 1 ? bf16hi(w[e / 2]) : bf16lo(w[e / 2]);
      const bool bad = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
      lo[e] = fminf(lo[e], bad ? -kMax : v);
      hi[e] = fmaxf(hi[e], bad ? kMax : v);
    }
  }
#pragma unroll
  for (int m = L; m < 64; m <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = fminf(lo[e], cpattn::shfl_xor_f(lo[e], m));
      hi[e] = fmaxf(hi[e], cpattn::shfl_xor_f(hi[e], m));
    }
  if (lane >= 2 * L) return;
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = lane < L ? pack(lo[2 * i], lo[2 * i + 1]) : pack(hi[2 * i], hi[2 * i + 1]);
  bounds[(blk * a.hkv + h) * 2 * L + lane] = make_uint4(o[0], o[1], o[2], o[3]);
}

template <int D, int B>
hipError_t launch_append_t(const AppendArgs& a, const AppendRows& rows, int n_rows, int tokens,
                           int v_items, hipStream_t s) {
  constexpr int HPW = 64 / (D / 8);
  // A wave's rotation serves about five loads of heads, or fewer where tokens are few.
  // us, 1 / 2 / 4 / 8 waves a token: 4,096 tokens on 32/8 heads of 128, ten loads, 29.7 /
  // 26.4 / 28.0 / -, on 64/8, eighteen, 50.5 / 40.7 / 40.4 / -, on 16/16 heads of 64, four,
  // 13.4 / 15.5 / 17.4; 1,024 tokens on 32/8 12.4 / 9.5 / 9.4 / 11.8, on 64/8 18.6 / 12.9 /
  // 11.8 / 13.9; 128 tokens on 64/8, 4 / 8 / 16: 7.0 / 5.8 / 6.3.
  const int groups = (a.hq + a.hkv + HPW - 1) / HPW;
  const int parts = std::max((groups + 4) / 5, (int)std::min<int64_t>(groups, (1024 + tokens - 1) / tokens));
  const int rope_blocks = (int)(((int64_t)tokens * parts + kWaves - 1) / kWaves);
  const int blocks = rope_blocks + (v_items + kWaves - 1) / kWaves;
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL((append_kernel<D, B>), dim3(blocks), dim3(kThreads), 0, s, r, a, tokens,
                       parts, rope_blocks, v_items, (const uint4*)a.qkv, (const uint4*)a.qw,
                       (const uint4*)a.kw, a.positions, a.bt, (uint4*)a.q, a.k_cache, a.v_cache);
  });
}

template <int D, int B>
hipError_t launch_bounds_t(const BoundsArgs& a, const BoundsRows& rows, int n_rows, int pages,
                           hipStream_t s) {
  const int items = pages * a.hkv;
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL((bounds_kernel<D, B>), dim3((items + kWaves - 1) / kWaves), dim3(kThreads),
                       0, s, r, a, items, a.k_cache, a.bt, (uint4*)a.bounds);
  });
}

template <int D, int B>
int v_items_t(int hkv) {
  return (hkv + VGeom<D, B>::HEADS - 1) / VGeom<D, B>::HEADS;
}

}  // namespace

int append_v_items(int d, int block, int hkv) {
  return d == 128 ? (block == 16 ? v_items_t<128, 16>(hkv) : v_items_t<128, 32>(hkv))
                  : (block == 16 ? v_items_t<64, 16>(hkv) : v_items_t<64, 32>(hkv));
}

hipError_t launch_append(int d, int block, const AppendArgs& a, const AppendRows& rows, int n_rows,
                         int tokens, int v_items, hipStream_t s) {
  auto f = d == 128 ? (block == 16 ? launch_append_t<128, 16> : launch_append_t<128, 32>)
                    : (block == 16 ? launch_append_t<64, 16> : launch_append_t<64, 32>);
  return f(a, rows, n_rows, tokens, v_items, s);
}

hipError_t launch_bounds(int d, int block, const BoundsArgs& a, const BoundsRows& rows, int n_rows,
                         int pages, hipStream_t s) {
  auto f = d == 128 ? (block == 16 ? launch_bounds_t<128, 16> : launch_bounds_t<128, 32>)
                    : (block == 16 ? launch_bounds_t<64, 16> : launch_bounds_t<64, 32>);
  return f(a, rows, n_rows, pages, s);
}

}  // namespace cpcache
