// Kernels of the attention over selected pages and behind common prefixes
// (cache_units.hpp has the work of a workgroup), and the merge.
#include "cache_units.hpp"

namespace cpcache {

namespace {

template <int D, int B, int NW, class Batch>
__global__ __launch_bounds__(64 * NW, 2) void pages_kernel(
    const Batch b, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt, const int32_t* __restrict__ pages) {
  constexpr int UNITS = NW == kWaves ? NW : 1;  // at most
  __shared__ __align__(16) uint8_t slices[NW][kSlice<D>];
  __shared__ Shared<NW> s;
  __shared__ int s_blocks[UNITS][kListPages], s_count[UNITS];
  token_units<D, B, true, NW>(b, (int)blockIdx.x, a, q, k_cache, v_cache, bt, pages, s, s_blocks,
                          s_count, [&](int w) { return slices[w]; });
}

// Tokens over all of their keys.
template <int D, int B, class Batch>
__global__ __launch_bounds__(64 * kAllWaves, 2) void tokens_kernel(
    const Batch b, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt) {
  __shared__ __align__(16) uint8_t slices[kAllWaves][kSlice<D>];
  __shared__ Shared<kAllWaves> s;
  token_units<D, B, false, kAllWaves>(b, (int)blockIdx.x, a, q, k_cache, v_cache, bt, nullptr, s,
                                      nullptr, nullptr, [&](int w) { return slices[w]; });
}

// The groups' workgroups come first, the tokens' behind them.
template <int D, int B, class Batch>
__global__ __launch_bounds__(kThreads, 2) void shared_kernel(
    const Batch b, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt) {
  __shared__ __align__(16) uint8_t slices[kWaves][kSlice<D>];
  __shared__ Shared<kWaves> s;
  const auto slice = [&](int w) { return slices[w]; };
  const int x = (int)blockIdx.x - a.group_items;
  if (x < 0) {
    const PrefixRow& row = b.g[row_index(b.g, &PrefixRow::item0, (int)blockIdx.x)];
    group_unit<D, B>(row, (int)blockIdx.x - row.item0, a, q, k_cache, v_cache, bt, s, slice);
    return;
  }
  token_units<D, B, false, kWaves>(b, x, a, q, k_cache, v_cache, bt, nullptr, s, nullptr, nullptr, slice);
}

// Merge of several pieces: with O_s and L_s, a piece's normalised output and the
// log2 of its weights' sum, the row's output is
//     sum_s 2^(L_s - max L) O_s / sum_s 2^(L_s - max L),
// over its own pieces and its group's.  A row (token, q head) takes `share` times
// D / 4 threads of 4 features, each of which takes every share-th piece; they meet
// in LDS.  A workgroup's rows are one token's.  3.1 us for a token of 4 pieces on 32
// heads; 6.4 for 128 tokens on 64 heads, 18 MB of partial rows: latency.
template <int D, int B, bool LIST, class Batch>
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(const Batch b, const AttnArgs a,
                                                               int per_token, int share) {
  constexpr int DQ = D / 4, SLOTS = merge_slots(D), U = 8;
  static_assert(SLOTS * DQ == kThreads, "merge_slots");
  __shared__ f32x4_t s_acc[SLOTS][DQ];
  __shared__ float s_m[SLOTS], s_w[SLOTS];
  const int64_t t = (int64_t)b.r[0].tok0 + (int)blockIdx.x / per_token;
  const Own row = own_of<B, LIST>(b, a, row_index(b.r, &AttnRow::tok0, (int)t));
  if (row.alone) return;
  const int slot = threadIdx.x / DQ, dq = threadIdx.x % DQ, per = SLOTS / share, p = slot / per;
  const int h = (int)blockIdx.x % per_token * per + slot % per;
  const int j = (int)(t - row.tok0), kvh = h >> a.log2_group, G = 1 << a.log2_group;
  const int e = h & (G - 1);
  float M = -INFINITY, W = 0.f;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  if (h < a.hq) {
    // unit (split, tokens, kvh) of the row's launch wrote their rows; pieces
    // [0, own) are the row's, those behind them the group's
    const int log2_rows = a.log2_tokens + a.log2_group, jb = j >> a.log2_tokens;
    const int64_t first = a.part0 + ((row.item0 + (int64_t)jb * a.hkv + kvh) << log2_rows) +
                          ((j - (jb << a.log2_tokens)) << a.log2_group) + e;
    const int64_t stride = (int64_t)(((row.n - 1) >> a.log2_tokens) + 1) * a.hkv << log2_rows;
    int own = row.n_split, n = own;
    int64_t gfirst = 0, gstride = 0;
    if (row.group >= 0) {
      const PrefixRow& g = b.g[row.group];
      gstride = (int64_t)g.n * G;
      gfirst = g.part0 + kvh * g.n_split * gstride + (t - g.tok0) * G + e;
      n += g.n_split;
    }
    for (int s0 = p; s0 < n; s0 += share * U) {
      float ls[U];
      f32x4_t o[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {  // past the last piece: it again, weight 0
        const int s = min(s0 + u * share, n - 1);
        const int64_t pr = s < own ? first + s * stride : gfirst + (s - own) * gstride;
        ls[u] = a.part_lse[pr];
        o[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + pr * D + dq * 4);
        if (s0 + u * share >= n) ls[u] = -INFINITY;
      }
      float m = M;
#pragma unroll
      for (int u = 0; u < U; ++u) m = fmaxf(m, ls[u]);
      const float keep = M == -INFINITY ? 0.f : exp2f(M - m);
      M = m;
      W *= keep;
      acc *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (ls[u] == -INFINITY) continue;
        const float w = exp2f(ls[u] - m);
        W += w;
        acc += w * o[u];
      }
    }
  }
  if (share > 1) {  // uniform
    s_acc[slot][dq] = acc;
    if (dq == 0) s_m[slot] = M, s_w[slot] = W;
    __syncthreads();
    if (p > 0) return;
    for (int k = 1; k < share; ++k) M = fmaxf(M, s_m[k * per + slot]);
    W = 0.f;
    acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < share; ++k) {
      const float wk = s_w[k * per + slot];
      if (wk == 0.f) continue;
      const float w = exp2f(s_m[k * per + slot] - M);
      W += w * wk;
      acc += w * s_acc[k * per + slot][dq];
    }
  }
  if (h >= a.hq) return;
  const float inv = W == 0.f ? 0.f : 1.f / W;
  *reinterpret_cast<uint2*>(a.out + (t * a.hq + h) * D + dq * 4) =
      make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
}

template <int D, int B>
hipError_t launch_pages_t(const AttnArgs& a, const AttnBatch& b, int n_rows, int items,
                          hipStream_t s) {
  return by_size(b, 0, n_rows, [&](const auto& x) {
    if (1 << a.log2_waves == kAllWaves)
      hipLaunchKernelGGL((pages_kernel<D, B, kAllWaves>), dim3(items), dim3(64 * kAllWaves), 0, s,
                         x, a, a.q, a.k_cache, a.v_cache, a.bt, a.pages);
    else
      hipLaunchKernelGGL((pages_kernel<D, B, kWaves>), dim3(items), dim3(kThreads), 0, s, x, a,
                         a.q, a.k_cache, a.v_cache, a.bt, a.pages);
  });
}

template <int D, int B>
hipError_t launch_shared_t(const AttnArgs& a, const AttnBatch& b, int n_rows, int items,
                           hipStream_t s) {
  return by_size(b, a.n_groups, n_rows, [&](const auto& x) {
    if (1 << a.log2_waves == kAllWaves)
      hipLaunchKernelGGL((tokens_kernel<D, B>), dim3(items), dim3(64 * kAllWaves), 0, s, x, a, a.q,
                         a.k_cache, a.v_cache, a.bt);
    else
      hipLaunchKernelGGL((shared_kernel<D, B>), dim3(items), dim3(kThreads), 0, s, x, a, a.q,
                         a.k_cache, a.v_cache, a.bt);
  });
}

template <int D, int B>
hipError_t launch_merge_t(const AttnArgs& a, const AttnBatch& b, int n_rows, int items,
                          int per_token, int share, hipStream_t s) {
  return by_size(b, a.n_groups, n_rows, [&](const auto& x) {
    if (a.pages)
      hipLaunchKernelGGL((cache_merge_kernel<D, B, true>), dim3(items), dim3(kThreads), 0, s, x, a,
                         per_token, share);
    else
      hipLaunchKernelGGL((cache_merge_kernel<D, B, false>), dim3(items), dim3(kThreads), 0, s, x,
                         a, per_token, share);
  });
}

}  // namespace

hipError_t launch_pages(int d, int block, const AttnArgs& a, const AttnBatch& b, int n_rows,
                        int items, hipStream_t s) {
  auto f = d == 128 ? (block == 16 ? launch_pages_t<128, 16> : launch_pages_t<128, 32>)
                    : (block == 16 ? launch_pages_t<64, 16> : launch_pages_t<64, 32>);
  return f(a, b, n_rows, items, s);
}

hipError_t launch_shared(int d, int block, const AttnArgs& a, const AttnBatch& b, int n_rows,
                         int items, hipStream_t s) {
  auto f = d == 128 ? (block == 16 ? launch_shared_t<128, 16> : launch_shared_t<128, 32>)
                    : (block == 16 ? launch_shared_t<64, 16> : launch_shared_t<64, 32>);
  return f(a, b, n_rows, items, s);
}

hipError_t launch_cache_merge(const cp_attn_desc& d, const AttnArgs& a, const AttnBatch& b,
                              int n_rows, int n_tokens, int most, hipStream_t s) {
  const int share = merge_share(d, n_tokens, most), items = (int)merge_items(d, n_tokens, share);
  const int per_token = (int)merge_items(d, 1, share);
  auto f = d.head_dim == 128 ? (d.block_size == 16 ? launch_merge_t<128, 16> : launch_merge_t<128, 32>)
                             : (d.block_size == 16 ? launch_merge_t<64, 16> : launch_merge_t<64, 32>);
  return f(a, b, n_rows, items, per_token, share, s);
}

}  // namespace cpcache
