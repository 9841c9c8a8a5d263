// Tree attention of many rows: the prefill tile (prefill_tile.inc, where its
// pipeline is described) with the mask of a drafted tree.
//
// A workgroup takes 32 NW of a kv head's rows, 32 a wave, and a piece of the
// key range, 64 keys at a time, K and V copied straight into LDS.  Steps that
// hold keys of the tree itself mask their scores by a 64-bit window of each
// row's mask and take infinities and NaN out of the V tile; those are noted,
// and the nodes that do see them get them added at the end.
#pragma once

#include "kernels.hpp"
#include "prefill_tile.hpp"
#include "tree_device.hpp"
#include "tree_plan.hpp"

namespace cptree {

struct TreeVis {
  static constexpr bool kTree = true;
  const uint64_t* mask;
  int words, n, first;  // nodes of the row, its first key of the tree
  unsigned long long* bad;

  __device__ __forceinline__ int start() const { return first; }
  __device__ __forceinline__ uint64_t seen(int t, int k0) const {
    return seen64(mask + (int64_t)t * words, words, n, k0 - first);
  }
  // the V tile of keys k0 .. k0 + 63 in LDS
  template <int D, int B, int NW>
  __device__ __forceinline__ void clean(uint8_t* vb, int k0, int tid) const {
    using L = cpattn::PrefillLayout<D, B>;
    constexpr int SLOTS = cpattn::BN / 8;  // 8 keys of a feature each
    for (int x = tid; x < SLOTS * D; x += NW * 64) {
      const int sl = x % SLOTS, d = x / SLOTS, k = k0 + sl * 8 - first;
      if (k + 8 <= 0) continue;
      uint32_t* p = reinterpret_cast<uint32_t*>(
          vb + (L::v_off(sl / (B / 8), d, sl % (B / 8)) - L::K_BYTES));
      uint32_t found = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t w = p[e];
        found |= clean_word(w, k + 2 * e, n) << (2 * e);
        p[e] = w;
      }
      note_bad(bad, found, k);
    }
  }
};

namespace {

using namespace cpattn;
using namespace cpattn::prefill_impl;

template <int D, int B, int G, int NW>
__global__ __launch_bounds__(NW * 64, 2) void wide_kernel(const TreeRows rows, const AttnArgs a) {
  constexpr int RG = 1;  // groups of 32 rows per wave
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
  __shared__ unsigned long long s_bad[kMaxWords];

  const TreeRow row = row_of(rows, blockIdx.x);
  constexpr int kNodes = 32 * NW / G;  // nodes per tile
  const int tiles = (row.n + kNodes - 1) / kNodes, units = row.n_split * a.hkv;
  // tiles of the same keys go to the same XCD: eight units at a time, tile by tile
  const int x = (int)blockIdx.x - row.item0;
  const int u0 = x / (8 * tiles) * 8, width = min(8, units - u0);
  const int y = x - u0 * tiles;
  const int unit = u0 + y % width, tile = y / width;
  const int kvh_ = unit % a.hkv, split = unit / a.hkv;
  const int ctx = row.start + row.n;
  PrefillRec it;
  it.tok0 = row.tok0 + tile * kNodes;
  it.n_tok = min(kNodes, row.n - tile * kNodes);
  it.pos0 = row.start;
  it.req = row.req;
  it.kv_begin = split * row.split_keys;
  it.kv_end = min(ctx, it.kv_begin + row.split_keys);
  it.part = row.n_split == 1
                ? -1
                : row.part0 + (kvh_ * row.n_split + split) * row.n * G + tile * kNodes * G;
  it.kvh = kvh_;
  if (threadIdx.x < kMaxWords) s_bad[threadIdx.x] = 0;
  __syncthreads();
  using Vis = TreeVis;
  const Vis vis{a.mask, a.words, row.n, row.start, s_bad};
  const uint16_t* q = a.q;
  const uint16_t* k_cache = a.k_cache;
  const uint16_t* v_cache = a.v_cache;
  const int32_t* bt = a.bt;
  uint16_t* out = a.out;
  float* part_o = a.part_o;
  float* part_lse = a.part_lse;
  const int hq = a.hq, hkv = a.hkv, mbr = a.mbr;
  const float scale_log2 = a.scale_log2;
  {
#include "prefill_tile.inc"
  }

  // ---- infinities and NaN that some node sees: rare, and not part of the tile
  __threadfence_block();
  __syncthreads();
  if (!(s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3])) return;
  for (int e = threadIdx.x; e < it.n_tok * G * D; e += NW * 64) {
    const int r = e / D, d = e % D;
    const int64_t t = it.tok0 + r / G;
    const float v = bad_values<D, B>(s_bad, a.mask + t * a.words, a.words, row, a, it.kvh, d);
    if (v == 0.f) continue;
    if (it.part < 0) {
      uint16_t* p = a.out + (t * a.hq + it.kvh * G + r % G) * D + d;
      *p = to_bf16(__uint_as_float((uint32_t)*p << 16) + v);
    } else {
      a.part_o[(int64_t)(it.part + r) * D + d] += v;
    }
  }
}

template <int D, int B, int G>
hipError_t launch_wide_w(int waves, const AttnArgs& a, const TreeRows& rows, int items,
                         hipStream_t s) {
  if (waves == 8)
    hipLaunchKernelGGL((wide_kernel<D, B, G, 8>), dim3(items), dim3(512), 0, s, rows, a);
  else
    hipLaunchKernelGGL((wide_kernel<D, B, G, 4>), dim3(items), dim3(256), 0, s, rows, a);
  return hipGetLastError();
}

template <int D, int B>
hipError_t launch_wide_g(int waves, const AttnArgs& a, const TreeRows& rows, int items,
                         hipStream_t s) {
  switch (a.log2_group) {
    case 0: return launch_wide_w<D, B, 1>(waves, a, rows, items, s);
    case 1: return launch_wide_w<D, B, 2>(waves, a, rows, items, s);
    case 2: return launch_wide_w<D, B, 4>(waves, a, rows, items, s);
    case 3: return launch_wide_w<D, B, 8>(waves, a, rows, items, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

}  // namespace cptree
