// Attention over selected pages and behind common prefixes (include/cp_cache.h).
//
// A decode token has G = Hq / Hkv rows per kv head for each key that is read, G
// flop a byte: its kernels are bound by the stream of K and V.  Tokens that
// share their keys bring G rows each.  All rows see all that their workgroup reads,
// up to the end of the range, but for neighbouring tokens of a row, each of which
// sees one key more than the one before: their last keys are masked column by column.
//
// Softmax runs in base 2, over one pass of the keys, with a running maximum
// that moves lazily (a score has to exceed it by 2^8).  The weights are rounded
// to bf16, the type that the matrix cores want beside V, and summed as rounded,
// in fp32.
#pragma once

#include "cache_device.hpp"
#include "cache_plan.hpp"

namespace cpcache {

using cpattn::bf16x8_t;
using cpattn::dot2_bf16;
using cpattn::f32x4_t;
using cpattn::kRescaleThreshold;
using cpattn::ld_global16;
using cpattn::ld_global16_nt;
using cpattn::pack_bf16x2;
using cpattn::shfl_xor_f;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ f32x4_t mfma16x16x32(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

template <int D>
constexpr int kSlice = 16 * D * 4;  // bytes of LDS per wave: 32 keys' rows, then 16 rows' output

// A wave's state over 16 NC rows, the columns of both products
// (v_mfma_f32_16x16x32_bf16), lane l = 16 g + i:
//   S^T (2 x 16 keys x 16 NC rows) = K . Q^T.  Row i of key half b is key
//     8 (i / 4) + 4 b + i % 4, so that lane (g, i) ends up with rows i's scores
//     of keys 8 g .. 8 g + 7, the B operand of the second product: the
//     weights never leave the lane.
//   O^T (D x 16 NC rows) += V^T . P^T: lane (g, i) reads 8 consecutive keys of
//     feature rows 16 dt + i, the A operand as the [D][B] blocks store it.
template <int D, int NC>
struct State {
  float m[NC], l[NC];
  f32x4_t o[NC][D / 16];
};

// Attends the wave's rows qv to keys [0, n_keys) of consecutive blocks, of which it
// takes tiles of 32 keys first, first + stride, ...; block_of(i) is the i-th block's
// place in the pool, for i below the blocks that n_keys fill.  The lane's column sees
// `mine` of the keys, and all columns see `least` (of an NC of 1; else all see all).
// Values that some do not see are taken out of the product where they are infinities
// or NaN, and added by those that do.  K and V are
// loaded as they lie in memory, K's rows passing through `slice`, LDS that only
// this wave uses.  K of the next tile is on its way from there on, V from the
// end of a tile to the product with it in the next.
//
// Bound by HBM where there is work for all CUs: 48 tokens on 64/8 heads of 128, 256
// pages of 16 each, 122 us for 807 MB, 6.6 TB/s.  One token's 64 pages, on 32/8 heads:
// 9.8 us by eight waves a kv head, a launch's latency and those of table, K, V, four
// tiles and the joining of the waves.
template <int D, int B, int NC, class BlockOf>
__device__ __forceinline__ void attend(State<D, NC>& st, const uint4 (&qv)[NC][D / 32], int n_keys,
                                       int mine, int least, int first, int stride, int kvh, int hkv, float scale_log2,
                                       const uint16_t* __restrict__ k_cache,
                                       const uint16_t* __restrict__ v_cache, uint8_t* slice,
                                       BlockOf&& block_of) {
  constexpr int TK = 32;         // keys per tile
  constexpr int NKS = D / 32;    // k-steps of a score
  constexpr int NDT = D / 16;    // 16-feature blocks of the output
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    st.m[c] = -INFINITY, st.l[c] = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) st.o[c][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (n_keys <= 0) return;
  const int64_t head_elems = (int64_t)B * D;
  const int n_tiles = (n_keys + TK - 1) / TK, last_block = (n_keys - 1) / B;
  const int voff = i * B + (8 * g) % B;
  const bool v_second = 8 * g >= B;
  constexpr int CH = D / 8, KPL = 64 / CH;  // 16-byte chunks per K row, rows per load
  constexpr int NKL = 16 / KPL;             // loads per half
  const int krow = lane / CH, kchunk = lane % CH;
  const int koff = (8 * (krow >> 2) + (krow & 3)) * D + kchunk * 8;
  auto slot = [](int r, int chunk) {
    return r * (D * 2) + ((chunk ^ (CH == 16 ? r & 15 : (r >> 1) & 7)) * 16);
  };
  // Each byte of K and V is read by one wave of the workgroup, so the loads are
  // non-temporal.  Other workgroups may read it, too: tokens of one prefix that each read
  // all of it (4.1 MB for 32 of them, in 10.8 us: 12 TB/s, from the caches all the same),
  // and further items of a row.  Past the range its last block comes again: those keys
  // are not seen.
  auto block_at = [&](int t, int second) {
    return ((int64_t)block_of(min(t * (TK / B) + second, last_block)) * hkv + kvh) * head_elems;
  };
  uint4 kr[2][NKL], vr[NDT];
  auto load_k = [&](int t) {
    const int64_t b0 = block_at(t, 0), b1 = B < TK ? block_at(t, 1) : b0;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < NKL; ++j) {
        const int key0 = 2 * KPL * j + 4 * b;  // the load's first key
        kr[b][j] = ld_global16_nt(k_cache + (key0 < B ? b0 : b1) + (key0 % B) * D + koff);
      }
  };
  auto load_v = [&](int t) {
    const int64_t b0 = block_at(t, 0), b1 = B < TK ? block_at(t, 1) : b0;
    const uint16_t* vp = v_cache + (v_second ? b1 : b0) + voff;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) vr[dt] = ld_global16_nt(vp + dt * 16 * B);
  };

  // tile t, with K of tile next requested on the way and V of it at the end
  auto step = [&](int t, int next) {
    f32x4_t s[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c) s[c][0] = s[c][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // a wave's LDS accesses complete in order: no wait but for the data
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < NKL; ++j)
        *reinterpret_cast<uint4*>(slice + b * 16 * D * 2 + slot(KPL * j + krow, kchunk)) =
            kr[b][j];
    load_k(next);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint4 k =
            *reinterpret_cast<const uint4*>(slice + b * 16 * D * 2 + slot(i, 4 * ks + g));
#pragma unroll
        for (int c = 0; c < NC; ++c) s[c][b] = mfma16x16x32(k, qv[c][ks], s[c][b]);
      }
    __builtin_amdgcn_wave_barrier();
    // the lane's values of keys from `end` on are zeroed
    const auto cut_v = [&](int end) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&vr[dt]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] &= (2 * e < end ? 0x0000ffffu : 0u) | (2 * e + 1 < end ? 0xffff0000u : 0u);
      }
    };
    const int left = n_keys - t * TK, all = least - t * TK;  // of the tile (wave-uniform)
    bool apart = false;  // values of keys from `all` on are added below
    if (all < TK) {  // those past the range may be anything, V included
      const int end = mine - t * TK - 8 * g;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= end) s[c][e >> 2][e & 3] = -INFINITY;
      cut_v(left - 8 * g);
      if constexpr (NC == 1) {
        if (all < left) {
          bool odd = false;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const uint32_t w[4] = {vr[dt].x, vr[dt].y, vr[dt].z, vr[dt].w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              odd |= 8 * g + e >= all && (w[e / 2] >> (16 * (e & 1)) & 0x7f80u) == 0x7f80u;
          }
          apart = __builtin_amdgcn_ballot_w64(odd) != 0;
          if (apart) cut_v(all - 8 * g);
        }
      }
    }
    uint4 pv[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float x = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])),
                      fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3]))) *
                scale_log2;
      if (__builtin_amdgcn_ballot_w64(x > st.m[c] + kRescaleThreshold)) {
        // the four lanes of a row share its maximum
        x = fmaxf(x, shfl_xor_f(x, 16));
        x = fmaxf(x, shfl_xor_f(x, 32));
        const float mnew = fmaxf(st.m[c], x);
        const float alpha = st.m[c] == -INFINITY ? 0.f : exp2f(st.m[c] - mnew);
        st.m[c] = mnew;
        st.l[c] *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) st.o[c][dt] *= alpha;
      }
      const float neg_m = st.m[c] == -INFINITY ? 0.f : -st.m[c];  // nothing seen yet
      uint32_t p[4];  // keys 8 g + 2 e, + 1
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[c][e >> 1][2 * (e & 1)], scale_log2, neg_m));
        const float p1 = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[c][e >> 1][2 * (e & 1) + 1], scale_log2, neg_m));
        p[e] = pack_bf16x2(p0, p1);
        st.l[c] = dot2_bf16(p[e], 0x3f803f80u, st.l[c]);  // the rounded weights
      }
      pv[c] = make_uint4(p[0], p[1], p[2], p[3]);
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int c = 0; c < NC; ++c) st.o[c][dt] = mfma16x16x32(vr[dt], pv[c], st.o[c][dt]);
    if constexpr (NC == 1) {
      if (apart)
        for (int k = max(all, 0); k < min(left, TK); ++k) {
          const uint32_t w[4] = {pv[0].x, pv[0].y, pv[0].z, pv[0].w};
          const uint32_t pair = k & 4 ? (k & 2 ? w[3] : w[2]) : (k & 2 ? w[1] : w[0]);
          const uint32_t theirs = __shfl(pair, 16 * (k >> 3) + i, 64);
          const float p = __uint_as_float(k & 1 ? theirs & 0xffff0000u : theirs << 16);
          const uint16_t* vp = v_cache + block_at(t, k / B) + k % B;
          if (t * TK + k < mine)
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                st.o[0][dt][r] +=
                    p * __uint_as_float((uint32_t)vp[(16 * dt + 4 * g + r) * B] << 16);
        }
    }
    load_v(next);
  };

  // The requests are unconditional (past the range its last tile again, which
  // is unused), so that the waits on them stay exact.
  const int last = n_tiles - 1;
  load_k(min(first, last));
  load_v(min(first, last));
  for (int t = first; t < n_tiles; t += stride) step(t, min(t + stride, last));
}

// The waves' states of up to kNarrowTile rows in LDS: row r of wave w counts with
// factor f[w][r] = 2^(m_w - max m) / (sum of all weights so scaled).
template <int NW>
struct Shared {
  float m[NW][kNarrowTile], l[NW][kNarrowTile], f[NW][kNarrowTile];
};

// The maxima and sums of `waves` waves from wave w0 on, which share 16 NC rows, and
// from them the rows' factors; x counts the threads of those waves.
// log_sum(row, y) gets the log2 of the sum of each row's weights.
template <int D, int NC, int NW, class LogSum>
__device__ __forceinline__ void join_waves(const State<D, NC>& st, Shared<NW>& s, int wave, int w0,
                                           int waves, int x, LogSum&& log_sum) {
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float l = st.l[c];
    l += shfl_xor_f(l, 16);
    l += shfl_xor_f(l, 32);
    if (g == 0) s.m[wave][16 * c + i] = st.m[c], s.l[wave][16 * c + i] = l;
  }
  __syncthreads();
  if (x < 16 * NC) {
    float M = -INFINITY, L = 0.f, m[NW], f[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      m[w] = w < waves ? s.m[w0 + w][x] : -INFINITY;
      f[w] = w < waves ? s.l[w0 + w][x] : 0.f;
      M = fmaxf(M, m[w]);
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float l = f[w];
      f[w] = m[w] == -INFINITY ? 0.f : exp2f(m[w] - M);
      L += f[w] * l;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;  // L == 0: it saw no key
#pragma unroll
    for (int w = 0; w < NW; ++w)
      if (w < waves) s.f[w0 + w][x] = f[w] * inv;
    log_sum(x, L == 0.f ? -INFINITY : M + __log2f(L));
  }
}

// Writes the sums of those waves' outputs, 16 rows at a time: put(row, p, v) gets
// features 4 p .. 4 p + 3 of each row below m_rows.  slice(w) is wave w's LDS.
template <int D, int NC, int NW, class Slice, class Put>
__device__ __forceinline__ void write_rows(const State<D, NC>& st, const Shared<NW>& s, int wave,
                                           int w0, int waves, int x0, int m_rows, Slice&& slice,
                                           Put&& put) {
  constexpr int NDT = D / 16;
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (16 * c >= m_rows) break;  // uniform
    __syncthreads();
    // lane (g, i) holds features 16 dt + 4 g .. + 3 of row i; 16-byte piece p
    // of row r lies at p ^ r, so that neither side meets a bank twice
    float* own = reinterpret_cast<float*>(slice(wave));
    if (16 * c + i < m_rows)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
        *reinterpret_cast<f32x4_t*>(own + i * D + ((4 * dt + g) ^ i) * 4) = st.o[c][dt];
    __syncthreads();
    for (int x = x0; x < 16 * (D / 4); x += 64 * waves) {
      const int p = x % (D / 4), r = x / (D / 4);
      if (16 * c + r >= m_rows) break;  // a thread's rows come in increasing order
      f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w)
        if (w < waves)
          v += s.f[w0 + w][16 * c + r] *
               *reinterpret_cast<const f32x4_t*>(
                   reinterpret_cast<const float*>(slice(w0 + w)) + r * D + (p ^ r) * 4);
      put(16 * c + r, p, v);
    }
  }
}

// A group's rows over a piece of its common keys.  A workgroup takes kNarrowTile
// (token, q head) rows of one kv head.
template <int D, int B, class Slice>
__device__ __forceinline__ void group_unit(const PrefixRow& row, int unit, const AttnArgs& a,
                                           const uint16_t* __restrict__ q,
                                           const uint16_t* __restrict__ k_cache,
                                           const uint16_t* __restrict__ v_cache,
                                           const int32_t* __restrict__ bt, Shared<kWaves>& s,
                                           Slice&& slice) {
  constexpr int NC = kNarrowTile / 16, NKS = D / 32;
  const int G = 1 << a.log2_group, all = row.n << a.log2_group;
  const int tiles = (all + kNarrowTile - 1) / kNarrowTile, m0 = unit % tiles * kNarrowTile;
  const int kvh = unit / tiles % a.hkv, split = unit / tiles / a.hkv;
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int begin = split * row.split_keys;
  const int n_keys = min(row.keys - begin, row.split_keys);
  uint4 qv[NC][NKS];
#pragma unroll
  for (int c = 0; c < NC; ++c) {  // past the last row that again (not stored)
    const int x = min(m0 + 16 * c + i, all - 1);
    const uint16_t* qb =
        q + (((int64_t)row.tok0 + (x >> a.log2_group)) * a.hq + kvh * G + (x & (G - 1))) * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qv[c][ks] = ld_global16(qb + ks * 32);
  }
  const int32_t* blocks = bt + (int64_t)row.req * a.mbr + begin / B;
  State<D, NC> st;
  attend<D, B, NC>(st, qv, n_keys, n_keys, n_keys, wave, kWaves, kvh, a.hkv, a.scale_log2, k_cache, v_cache,
                   slice(wave), [&](int b) { return blocks[b]; });
  const int64_t part = (int64_t)row.part0 + ((int64_t)kvh * row.n_split + split) * all + m0;
  join_waves(st, s, wave, 0, kWaves, threadIdx.x, [&](int r, float x) {
    if (m0 + r < all) a.part_lse[part + r] = x;
  });
  write_rows(st, s, wave, 0, kWaves, threadIdx.x, min(kNarrowTile, all - m0), slice,
             [&](int r, int p, const f32x4_t& v) {
               *reinterpret_cast<f32x4_t*>(a.part_o + (part + r) * D + 4 * p) = v;
             });
}

// What a workgroup or a merge needs of row r of a launch.
struct Own {
  int32_t tok0, n, start, req, item0;
  int group;    // the launch's, or -1
  int keys;     // that are read for the group
  int n_split;
  bool alone;   // one piece in all: its workgroup writes the output
};

template <int B, bool LIST, class Batch>
__device__ __forceinline__ Own own_of(const Batch& b, const AttnArgs& a, int r) {
  const AttnRow row = b.r[r];
  Own o{row.tok0, b.r[r + 1].tok0 - row.tok0, row.start, row.req, row.item0, -1, 0, 1, true};
  if constexpr (!LIST) {
    constexpr int NG = sizeof(b.g) / sizeof(PrefixRow);
    static_assert(NG <= 64, "a group per lane");
    const int lane = threadIdx.x & 63, g = min(lane, NG - 1);
    const uint64_t in = __builtin_amdgcn_ballot_w64(lane < a.n_groups && b.g[g].row0 <= r &&
                                                    r < b.g[g].row1);
    if (in) {
      o.group = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)in) - 1);
      o.keys = b.g[o.group].keys;
    }
  }
  const int last = o.start + o.n - 1;
  const int own = LIST ? min(a.n_pages, last / B + 1) : last + 1 - o.keys;
  o.n_split = (own - 1) / a.piece + 1;
  o.alone = o.n_split == 1 && o.group < 0;
  return o;
}

// A workgroup of tokens: each of its units, taken by 2^a.log2_waves waves or by all
// kAllWaves, are the G rows of up to 2^a.log2_tokens tokens of a row (the columns, 16 at
// most) over a piece of their own keys, or (LIST) of one token over a piece of its page
// list, whose blocks come to s_blocks, their number to s_count.  Tokens taken together
// read K and V once: 128 rows of up to 4 tokens behind ~500 keys of their own, 64/8 heads
// of 128, 148 -> 112 us; 266 rows of a dozen keys, 16/16 heads of 64, 48 -> 35.
template <int D, int B, bool LIST, int NW, class Batch, class Slice>
__device__ __forceinline__ void token_units(const Batch& b, int block, const AttnArgs& a,
                                            const uint16_t* __restrict__ q,
                                            const uint16_t* __restrict__ k_cache,
                                            const uint16_t* __restrict__ v_cache,
                                            const int32_t* __restrict__ bt,
                                            const int32_t* __restrict__ pages, Shared<NW>& s,
                                            int (*s_blocks)[kListPages], int* s_count,
                                            Slice&& slice) {
  constexpr int NKS = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int log2_waves = NW == kWaves ? a.log2_waves : __builtin_ctz(NW);
  const int W = 1 << log2_waves, mine = wave >> log2_waves, w0 = mine << log2_waves;
  const int x = tid - 64 * w0, item = block * (NW >> log2_waves) + mine;
  const bool real = item < a.items;  // the last workgroup may have fewer units
  const Own row = own_of<B, LIST>(b, a, row_index(b.r, &AttnRow::item0, min(item, a.items - 1)));
  const int unit = min(item, a.items - 1) - row.item0;
  const int G = 1 << a.log2_group, log2_tokens = LIST ? 0 : a.log2_tokens;
  const int blocks_of = LIST ? row.n : ((row.n - 1) >> log2_tokens) + 1;
  const int kvh = unit % a.hkv, split = unit / a.hkv / blocks_of;
  const int j = (unit / a.hkv % blocks_of) << log2_tokens;  // the first token
  const int rows = min(1 << log2_tokens, row.n - j) << a.log2_group;
  const int64_t t = (int64_t)row.tok0 + j;
  const int pos = row.start + j;
  const int32_t* bt_row = bt + (int64_t)row.req * a.mbr;
  uint4 qv[1][NKS];
  const int col = min(i, rows - 1);  // past the last row that again (not stored)
  {
    const uint16_t* qb =
        q + ((t + (col >> a.log2_group)) * a.hq + kvh * G + (col & (G - 1))) * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qv[0][ks] = ld_global16(qb + ks * 32);
  }
  State<D, 1> st;
  int n_keys = 0;
  if constexpr (LIST) {
    // the piece's entries that count, and their blocks
    const int e0 = split * a.piece, e1 = min(a.n_pages, e0 + a.piece), top = pos / B;
    const int32_t* list = pages + (t * a.hkv + kvh) * a.n_pages;
    if (x == 0) s_count[mine] = e1;
    __syncthreads();
    for (int e = x; e < e1; e += 64 * W) {
      const int page = list[e], before = e > 0 ? list[e - 1] : -1;
      if (page < 0 || page <= before || page > top) atomicMin(&s_count[mine], e);
      else if (e >= e0) s_blocks[mine][e - e0] = bt_row[page];
    }
    __syncthreads();
    const int end = s_count[mine], count = end - e0;
    if (count > 0) {  // only the last entry's page can be p's own
      n_keys = count * B;
      if (list[end - 1] == top) n_keys -= B - 1 - pos % B;
    }
    const int* blocks = s_blocks[mine];
    if (!real) n_keys = 0;
    attend<D, B, 1>(st, qv, n_keys, n_keys, n_keys, wave - w0, W, kvh, a.hkv, a.scale_log2,
                    k_cache, v_cache, slice(wave),
                    [&](int b) { return __builtin_amdgcn_readfirstlane(blocks[b]); });
  } else {
    const int64_t begin = row.keys + (int64_t)split * a.piece;
    const auto seen = [&](int ahead) {  // by the token so far behind the first one; maybe none
      return (int)min((int64_t)a.piece, pos + ahead + 1 - begin);
    };
    n_keys = real ? seen((rows - 1) >> a.log2_group) : 0;
    const int32_t* blocks = bt_row + begin / B;
    attend<D, B, 1>(st, qv, n_keys, seen(col >> a.log2_group), seen(0), wave - w0, W, kvh, a.hkv,
                    a.scale_log2, k_cache, v_cache, slice(wave),
                    [&](int b) { return blocks[b]; });
  }
  const int64_t part =
      (int64_t)a.part0 + (((int64_t)row.item0 + unit) << (log2_tokens + a.log2_group));
  join_waves(st, s, wave, w0, W, x, [&](int r, float y) {
    if (real && !row.alone && r < rows) a.part_lse[part + r] = y;
  });
  // (all units of the workgroup write as many rows as a unit can have: the same barriers)
  write_rows(st, s, wave, w0, W, x, G << log2_tokens, slice, [&](int r, int p, const f32x4_t& v) {
    if (!real || r >= rows) return;
    if (row.alone)
      *reinterpret_cast<uint2*>(a.out +
                                ((t + (r >> a.log2_group)) * a.hq + kvh * G + (r & (G - 1))) * D +
                                4 * p) =
          make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    else
      *reinterpret_cast<f32x4_t*>(a.part_o + (part + r) * D + 4 * p) = v;
  });
}

}  // namespace

}  // namespace cpcache
