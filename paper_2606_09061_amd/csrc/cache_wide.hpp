// Attention of many rows to the keys that they have in common: the prefill tile
// (prefill_tile.inc, where its pipeline is described) without a mask.
//
// A workgroup takes 128 of a kv head's rows, 32 a wave, and a piece of the common
// keys, 64 at a time, K and V copied straight into LDS.  Every row sees all of
// them, but for the end of the range.  Groups of few rows and the tokens' own keys
// have workgroups of their own (cache_units.hpp) in the same launch.
//
// 8 groups of 16 requests, ~4,100 keys in common and ~300 of their own, 64/8 heads of
// 128: 66.5 us for 323 MB, 4.9 TB/s, bound by HBM.  One group of 32 requests and ~8,200
// keys, 32/8: 19.0 us for 58 MB: 176 workgroups of six steps, 0.85 us each behind 14 us of
// launch, first loads and stores.
#pragma once

#include "cache_units.hpp"
#include "kernels.hpp"
#include "prefill_tile.hpp"

namespace cpcache {

struct PrefixVis {
  static constexpr bool kTree = true;  // steps past start() ask for what is seen
  int end;

  __device__ __forceinline__ int start() const { return end; }
  // of the keys from k0 on
  __device__ __forceinline__ uint64_t seen(int, int k0) const {
    const int n = end - k0;
    return n >= 64 ? ~0ull : n <= 0 ? 0 : (1ull << n) - 1;
  }
  // the V tile of keys k0 .. k0 + 63 in LDS: whole pages are past the end or not
  template <int D, int B, int NW>
  __device__ __forceinline__ void clean(uint8_t* vb, int k0, int tid) const {
    using L = cpattn::PrefillLayout<D, B>;
    constexpr int SLOTS = cpattn::BN / 8;  // 8 keys of a feature each
    for (int x = tid; x < SLOTS * D; x += NW * 64) {
      const int sl = x % SLOTS, d = x / SLOTS;
      if (k0 + sl * 8 < end) continue;
      *reinterpret_cast<uint4*>(vb + (L::v_off(sl / (B / 8), d, sl % (B / 8)) - L::K_BYTES)) =
          make_uint4(0, 0, 0, 0);
    }
  }
};

namespace {

using namespace cpattn;
using namespace cpattn::prefill_impl;
using cpcache::AttnArgs;  // not cpattn's

// prefill_impl::copy16_to_lds past the caches, for keys that one workgroup reads
__device__ __forceinline__ void copy16_to_lds_nt(const uint16_t* base, uint32_t byte_off,
                                                 uint8_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t dst = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(byte_off), "s"(base),
               "{m0}"(dst)
               : "memory");
#endif
}

// The pointers come as arguments of their own, which may be restrict: the table's
// entries are then scalar loads, and no wait for one drains the copies on their way.
template <int D, int B, int G>
__global__ __launch_bounds__(2 * kWideTile, 2) void shared_wide_kernel(
    const AttnBatch b, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt, uint16_t* __restrict__ out, float* __restrict__ part_o,
    float* __restrict__ part_lse) {
  constexpr int NW = kWideTile / 32, RG = 1;  // waves, groups of 32 rows of each
  using C = PrefillGeom<D, B, NW>;
  using L = PrefillLayout<D, B>;
  constexpr int NKS = C::NKS, NDT = C::NDT, NQK = C::NQK, NPV = C::NPV, PW = C::PW;
  constexpr int KCH = C::KCH, NBW = C::NBW, kRing = C::kRing;
  constexpr int NP = 16 * RG;  // weight pairs per lane and step
  using T_ = std::true_type;
  using F_ = std::false_type;
  __shared__ __attribute__((aligned(1024))) uint8_t kb0[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t kb1[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t vb0[C::TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t vb1[C::TILE_BYTES];

  __shared__ Shared<kWaves> s;
  // a wave's slice, half a tile
  const auto slice = [&](int w) {
    static_assert(2 * kSlice<D> == C::TILE_BYTES, "slices");
    return (w < 2 ? kb0 : kb1) + (w & 1) * kSlice<D>;
  };
  const int token_item = (int)blockIdx.x - a.group_items;
  if (token_item >= 0) {
    token_units<D, B, false, kWaves>(b, token_item, a, q, k_cache, v_cache, bt, nullptr, s, nullptr,
                             nullptr, slice);
    return;
  }
  const PrefixRow& row = b.g[row_index(b.g, &PrefixRow::item0, (int)blockIdx.x)];
  if (!row.wide) {
    group_unit<D, B>(row, (int)blockIdx.x - row.item0, a, q, k_cache, v_cache, bt, s, slice);
    return;
  }
  constexpr int kTokens = kWideTile / G;  // per tile
  const int tiles = (row.n + kTokens - 1) / kTokens, units = row.n_split * a.hkv;
  // tiles of the same keys go to the same XCD: eight units at a time, tile by tile
  const int x = (int)blockIdx.x - row.item0;
  const int u0 = x / (8 * tiles) * 8, width = min(8, units - u0);
  const int y = x - u0 * tiles;
  const int unit = u0 + y % width, tile = y / width;
  const int kvh_ = unit % a.hkv, split = unit / a.hkv;
  PrefillRec it;
  it.tok0 = row.tok0 + tile * kTokens;
  it.n_tok = min(kTokens, row.n - tile * kTokens);
  it.pos0 = row.keys;
  it.req = row.req;
  it.kv_begin = split * row.split_keys;
  it.kv_end = min(row.keys - it.kv_begin, row.split_keys) + it.kv_begin;
  it.part = row.part0 + (kvh_ * row.n_split + split) * row.n * G + tile * kTokens * G;
  it.kvh = kvh_;
  using Vis = PrefixVis;
  const Vis vis{it.kv_end};
  const int hq = a.hq, hkv = a.hkv, mbr = a.mbr;
  const float scale_log2 = a.scale_log2;
  // what the tile copies K and V with
  const bool streamed = row.wide == kStreamed;
  const auto copy16_to_lds = [&](const uint16_t* base, uint32_t byte_off, uint8_t* lds) {
    if (streamed) copy16_to_lds_nt(base, byte_off, lds);
    else prefill_impl::copy16_to_lds(base, byte_off, lds);
  };
#include "prefill_tile.inc"
}

template <int D, int B>
hipError_t launch_shared_wide_g(const AttnArgs& a, const AttnBatch& b, int items,
                                hipStream_t s) {
  auto kern = a.log2_group == 0   ? shared_wide_kernel<D, B, 1>
              : a.log2_group == 1 ? shared_wide_kernel<D, B, 2>
              : a.log2_group == 2 ? shared_wide_kernel<D, B, 4>
                                  : shared_wide_kernel<D, B, 8>;
  hipLaunchKernelGGL(kern, dim3(items), dim3(2 * kWideTile), 0, s, b, a, a.q, a.k_cache,
                     a.v_cache, a.bt, a.out, a.part_o, a.part_lse);
  return hipGetLastError();
}

}  // namespace

}  // namespace cpcache
