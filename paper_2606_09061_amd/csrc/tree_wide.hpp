// Tree attention of many rows: the prefill tile (prefill_tile.inc, where its
// pipeline is described) with the mask of a drafted tree.
//
// A workgroup takes 128 of a kv head's rows, 32 a wave, and a piece of the
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
  const uint64_t (*mask)[kMaxWords];  // of the tile's nodes, in LDS
  int words, n, first;                // nodes of the row, its first key of the tree
  unsigned long long* bad;

  __device__ __forceinline__ int start() const { return first; }
  // of the tile's node `node`, the keys from k0 on
  __device__ __forceinline__ uint64_t seen(int node, int k0) const {
    return seen64(mask[node], words, n, k0 - first);
  }
  // the V tile of keys k0 .. k0 + 63 in LDS
  template <int D, int B, int NW>
  __device__ __forceinline__ void clean(uint8_t* vb, int k0, int tid) const {
    using L = cpattn::PrefillLayout<D, B>;
    constexpr int SLOTS = cpattn::BN / 8;  // 8 keys of a feature each
    for (int x = tid; x < SLOTS * D; x += NW * 64) {
      const int sl = x % SLOTS, d = x / SLOTS, k = k0 + sl * 8 - first;
      if (k + 8 <= 0) continue;
      uint4* p = reinterpret_cast<uint4*>(
          vb + (L::v_off(sl / (B / 8), d, sl % (B / 8)) - L::K_BYTES));
      uint32_t w[4] = {p->x, p->y, p->z, p->w}, found = 0;
      u16x2_t top = {0, 0};  // of the values without their signs
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, w[e] & 0x7fff7fffu));
      if (k + 8 <= n && max(top[0], top[1]) < 0x7f80) continue;  // as it should be
#pragma unroll
      for (int e = 0; e < 4; ++e) found |= clean_word(w[e], k + 2 * e, n) << (2 * e);
      *p = make_uint4(w[0], w[1], w[2], w[3]);
      note_bad(bad, found, k);
    }
  }
};

namespace {

using namespace cpattn;
using namespace cpattn::prefill_impl;

// The pointers come as arguments of their own, which may be restrict: the table's
// entries are then scalar loads, and no wait for one drains the copies on their
// way (24 requests of up to 64 nodes 161 -> 133 us).
template <int D, int B, int G>
__global__ __launch_bounds__(2 * kWideRows, 2) void wide_kernel(
    const TreeRows rows, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt, uint16_t* __restrict__ out, float* __restrict__ part_o,
    float* __restrict__ part_lse) {
  constexpr int NW = kWideRows / 32, RG = 1;  // waves, groups of 32 rows of each
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
  __shared__ uint64_t s_mask[kWideRows / G][kMaxWords];

  const TreeRow row = row_of(rows, blockIdx.x);
  constexpr int kNodes = kWideRows / G;  // nodes per tile
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
  if (it.kv_end > row.start)  // some of the tree's own keys
    for (int e = threadIdx.x; e < it.n_tok * a.words; e += 2 * kWideRows)
      s_mask[e / a.words][e % a.words] = a.mask[(int64_t)it.tok0 * a.words + e];
  __syncthreads();
  using Vis = TreeVis;
  const Vis vis{s_mask, a.words, row.n, row.start, s_bad};
  const int hq = a.hq, hkv = a.hkv, mbr = a.mbr;
  const float scale_log2 = a.scale_log2;
  {
#include "prefill_tile.inc"
  }

  // ---- infinities and NaN that some node sees: rare, and not part of the tile
  if (!(s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3])) return;  // complete since the last step
  __threadfence_block();
  __syncthreads();  // the tile's rows are written
  for (int e = threadIdx.x; e < it.n_tok * G * D; e += 2 * kWideRows) {
    const int r = e / D, d = e % D;
    const int64_t t = it.tok0 + r / G;
    const float v = bad_values<D, B>(s_bad, a.mask + t * a.words, a.words, row, a, it.kvh, d);
    if (v == 0.f) continue;
    if (it.part < 0) {
      uint16_t* p = out + (t * a.hq + it.kvh * G + r % G) * D + d;
      *p = to_bf16(__uint_as_float((uint32_t)*p << 16) + v);
    } else {
      part_o[(int64_t)(it.part + r) * D + d] += v;
    }
  }
}

template <int D, int B>
hipError_t launch_wide_g(const AttnArgs& a, const TreeRows& rows, int items, hipStream_t s) {
  auto kern = a.log2_group == 0   ? wide_kernel<D, B, 1>
              : a.log2_group == 1 ? wide_kernel<D, B, 2>
              : a.log2_group == 2 ? wide_kernel<D, B, 4>
                                  : wide_kernel<D, B, 8>;
  hipLaunchKernelGGL(kern, dim3(items), dim3(2 * kWideRows), 0, s, rows, a, a.q, a.k_cache,
                     a.v_cache, a.bt, a.out, a.part_o, a.part_lse);
  return hipGetLastError();
}

}  // namespace

}  // namespace cptree
