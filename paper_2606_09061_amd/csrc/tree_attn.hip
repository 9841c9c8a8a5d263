// Attention of drafted trees over the paged cache (include/cp_tree.h): the
// narrow kernel and the merge (tree_wide.hpp has the wide one).
//
// With n nodes and G q heads per kv head, n G rows share every K and V that
// is read.  Over c committed keys the work is 4 D n G c flop on 4 D c bytes per
// kv head, n G flop a byte: up to some 150 rows the stream of K and V bounds
// it, above that the matrix cores.
//
// Softmax runs in base 2, over one pass of the keys, with a running maximum
// that moves lazily (a score has to exceed it by 2^8).  The weights are rounded
// to bf16, the type that the matrix cores want beside V; exact products would
// need a second one with what the rounding leaves.  fp32 sums of the weights as
// rounded keep the rows normalised: outputs are off by 0.0022 to 0.0023 in the
// mean square against 0.0016 to 0.0017 of their own rounding, as in the mixed
// step.  Masks cost nothing until the keys of the tree itself, the last ones of
// a row.
#include "tree_attn.hpp"

#include "tree_device.hpp"
#include "tree_plan.hpp"

namespace cptree {

using cpattn::bf16x8_t;
using cpattn::dot2_bf16;
using cpattn::f32x4_t;
using cpattn::kRescaleThreshold;
using cpattn::ld_global16;
using cpattn::ld_global16_nt;
using cpattn::pack_bf16x2;
using cpattn::shfl_xor_f;
using cpattn::to_bf16;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ f32x4_t mfma16x16x32(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// A workgroup takes 16 NC of a kv head's rows and a piece of the key range, of
// which wave w takes tiles of 32 keys w, w + 4, ...  (With one such tile of rows
// the stream of K and V bounds it: 32 requests of 8 nodes on 32/8 heads, 206 MB,
// 38 us or 5.4 TB/s.)  The rows are the columns of both products
// (v_mfma_f32_16x16x32_bf16, NC of them per operand of K or V).  Per tile and
// wave, lane l = 16 g + i:
//   S^T (2 x 16 keys x 16 NC rows) = K . Q^T.  Row i of key half b is key
//     8 (i / 4) + 4 b + i % 4, so that lane (g, i) ends up with rows i's scores
//     of keys 8 g .. 8 g + 7, the B operand of the second product: the
//     weights never leave the lane.
//   O^T (D x 16 NC rows) += V^T . P^T: lane (g, i) reads 8 consecutive keys of
//     feature rows 16 dt + i, the A operand as the [D][B] blocks store it.
// K and V are loaded as they lie in memory, K's rows passing through a slice
// of LDS that only this wave uses.  K of the next tile is on its way from
// there on, V from the end of a tile to the product with it in the next.  The
// waves' states are combined in LDS, 16 rows at a time.
//
// V of the tree's own keys enters the product with infinities and NaN as
// zeros: a node that does not see the key would get 0 * NaN from it.  The
// nodes that do get them added at the end.
template <int D, int B, int NC, class Rows>
__global__ __launch_bounds__(kThreads, 2) void narrow_kernel(
    const Rows rows, const AttnArgs a, const uint16_t* __restrict__ q,
    const uint16_t* __restrict__ k_cache, const uint16_t* __restrict__ v_cache,
    const int32_t* __restrict__ bt, const uint64_t* __restrict__ masks) {
  constexpr int TK = 32;       // keys per tile
  constexpr int ROWS = 16 * NC;
  constexpr int NKS = D / 32;    // k-steps of a score
  constexpr int NDT = D / 16;    // 16-feature blocks of the output
  constexpr int SLICE = 16 * D * 4;  // bytes of a wave: 32 keys' rows, then 16 rows' output
  __shared__ __align__(16) uint8_t slices[kWaves][SLICE];
  __shared__ float s_m[kWaves][ROWS], s_l[kWaves][ROWS], s_f[kWaves][ROWS];
  __shared__ unsigned long long s_bad[kMaxWords];

  const TreeRow row = row_of(rows, blockIdx.x);
  const int unit = (int)blockIdx.x - row.item0;
  const int G = 1 << a.log2_group, m_rows = row.n << a.log2_group;
  const int tiles = (m_rows + ROWS - 1) / ROWS, m0 = unit % tiles * ROWS;
  const int kvh = unit / tiles % a.hkv, split = unit / tiles / a.hkv;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ctx = row.start + row.n;
  const int kv_begin = split * row.split_keys, kv_end = min(ctx, kv_begin + row.split_keys);
  if (tid < kMaxWords) s_bad[tid] = 0;

  // Column c's row of this lane, past the last one that again (not stored), and
  // its node's mask, one word.
  uint4 qv[NC][NKS];
  uint64_t mask[NC];
  static_assert(kNarrowNodes <= 64, "one word");
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int x = min(m0 + 16 * c + i, m_rows - 1);
    const int64_t t = row.tok0 + (x >> a.log2_group);
    const uint16_t* qb = q + (t * a.hq + kvh * G + (x & (G - 1))) * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qv[c][ks] = ld_global16(qb + ks * 32);
    mask[c] = masks[t * a.words];
  }
  __builtin_amdgcn_sched_barrier(0);

  float m_run[NC], l_run[NC];
  f32x4_t o[NC][NDT];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m_run[c] = -INFINITY, l_run[c] = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[c][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  const int64_t head_elems = (int64_t)B * D;
  const int32_t* bt_row = bt + (int64_t)row.req * a.mbr;
  const int n_tiles = (kv_end - kv_begin + TK - 1) / TK;
  const int lb_last = (kv_end - 1) / B;
  const int voff = i * B + (8 * g) % B;
  const bool v_second = 8 * g >= B;
  constexpr int CH = D / 8, KPL = 64 / CH;  // 16-byte chunks per K row, rows per load
  constexpr int NKL = 16 / KPL;             // loads per half
  const int krow = lane / CH, kchunk = lane % CH;
  const int koff = (8 * (krow >> 2) + (krow & 3)) * D + kchunk * 8;
  uint8_t* slice = slices[wave];
  auto slot = [](int r, int chunk) {
    return r * (D * 2) + ((chunk ^ (CH == 16 ? r & 15 : (r >> 1) & 7)) * 16);
  };
  // Each byte of K and V is read by one wave of the workgroup: streamed past the
  // caches.
  // Past the range its last block comes again: those keys are not seen.
  auto block_at = [&](int t, int second) {
    const int lb = min(kv_begin / B + t * (TK / B) + second, lb_last);
    return ((int64_t)bt_row[lb] * a.hkv + kvh) * head_elems;
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
    const int k0 = kv_begin + t * TK;
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
    if (k0 + TK > row.start) {  // the tree's own keys (wave-uniform)
      const int o0 = k0 - row.start, first = o0 + 8 * g;  // tree offsets: tile's, this lane's
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint64_t m = row.n < 64 ? mask[c] & ((1ull << row.n) - 1) : mask[c];
        m = o0 >= 64 ? 0 : o0 >= 0 ? m >> o0 : m << -o0 | ((1ull << -o0) - 1);
        const uint32_t seen = (uint32_t)m >> (8 * g);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(seen >> e & 1)) s[c][e >> 2][e & 3] = -INFINITY;
      }
      // keys past the row, whose slots may hold anything
      uint32_t keep[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        keep[e] = (first + 2 * e < row.n ? 0x0000ffffu : 0u) |
                  (first + 2 * e + 1 < row.n ? 0xffff0000u : 0u);
      u16x2_t top = {0, 0};  // of the values without their signs
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&vr[dt]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] &= keep[e];
          top = __builtin_elementwise_max(top,
                                          __builtin_bit_cast(u16x2_t, w[e] & 0x7fff7fffu));
        }
      }
      if (__builtin_amdgcn_ballot_w64(max(top[0], top[1]) >= 0x7f80)) {
        // rare: one word at a time, in the slice that K no longer needs
        uint4* own = reinterpret_cast<uint4*>(slice) + lane;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) own[64 * dt] = vr[dt];
        uint32_t found = 0;
#pragma unroll 1
        for (int x = 0; x < 4 * NDT; ++x) {
          uint32_t* w = reinterpret_cast<uint32_t*>(own + 64 * (x >> 2)) + (x & 3);
          uint32_t v = *w;
          found |= clean_word(v, first + 2 * (x & 3), row.n) << (2 * (x & 3));
          *w = v;
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) vr[dt] = own[64 * dt];
        note_bad(s_bad, found, first);
      }
    }
    uint4 pv[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float x = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])),
                      fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3]))) *
                a.scale_log2;
      if (__builtin_amdgcn_ballot_w64(x > m_run[c] + kRescaleThreshold)) {
        // the four lanes of a row share its maximum
        x = fmaxf(x, shfl_xor_f(x, 16));
        x = fmaxf(x, shfl_xor_f(x, 32));
        const float mnew = fmaxf(m_run[c], x);
        const float alpha = m_run[c] == -INFINITY ? 0.f : exp2f(m_run[c] - mnew);
        m_run[c] = mnew;
        l_run[c] *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[c][dt] *= alpha;
      }
      const float neg_m = m_run[c] == -INFINITY ? 0.f : -m_run[c];  // nothing seen yet
      uint32_t p[4];  // keys 8 g + 2 e, + 1
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[c][e >> 1][2 * (e & 1)], a.scale_log2, neg_m));
        const float p1 = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s[c][e >> 1][2 * (e & 1) + 1], a.scale_log2, neg_m));
        p[e] = pack_bf16x2(p0, p1);
        l_run[c] = dot2_bf16(p[e], 0x3f803f80u, l_run[c]);  // the rounded weights
      }
      pv[c] = make_uint4(p[0], p[1], p[2], p[3]);
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c][dt] = mfma16x16x32(vr[dt], pv[c], o[c][dt]);
    load_v(next);
  };

  __syncthreads();  // s_bad is clear
  {
    // The requests are unconditional (past the range its last tile again,
    // which is unused), so that the waits on them stay exact.
    const int last = n_tiles - 1;  // a piece is never empty
    load_k(min(wave, last));
    load_v(min(wave, last));
    for (int t = wave; t < n_tiles; t += kWaves) step(t, min(t + kWaves, last));
  }

  // ---- combine the waves and write: wave w's row r counts with factor
  // s_f[w][r] = 2^(m_w - max m) / (sum of the waves' sums so weighted)
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float l = l_run[c];
    l += shfl_xor_f(l, 16);
    l += shfl_xor_f(l, 32);
    if (g == 0) s_m[wave][16 * c + i] = m_run[c], s_l[wave][16 * c + i] = l;
  }
  __syncthreads();
  const int64_t part0 =
      (int64_t)row.part0 + ((int64_t)kvh * row.n_split + split) * m_rows;
  if (tid < ROWS) {
    float M = -INFINITY, L = 0.f, f[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][tid]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float m = s_m[w][tid];
      f[w] = m == -INFINITY ? 0.f : exp2f(m - M);
      L += f[w] * s_l[w][tid];
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;  // L == 0: it saw no key
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s_f[w][tid] = f[w] * inv;
    if (row.n_split > 1 && m0 + tid < m_rows)
      a.part_lse[part0 + m0 + tid] = L == 0.f ? -INFINITY : M + __log2f(L);
  }
  const uint64_t any = s_bad[0];
  auto red = reinterpret_cast<float(*)[16][D]>(&slices[0][0]);
  static_assert(sizeof(float) * 16 * D == SLICE, "a wave's output fills its slice");
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (m0 + 16 * c >= m_rows) break;  // uniform
    __syncthreads();
    // lane (g, i) holds features 16 dt + 4 g .. + 3 of row i; 16-byte piece p
    // of row r lies at p ^ r, so that neither side meets a bank twice
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
      *reinterpret_cast<f32x4_t*>(&red[wave][i][((4 * dt + g) ^ i) * 4]) = o[c][dt];
    __syncthreads();
    for (int x = tid; x < 16 * (D / 4); x += kThreads) {
      const int p = x % (D / 4), r = x / (D / 4), mr = m0 + 16 * c + r;
      if (mr >= m_rows) break;  // a thread's rows come in increasing order
      f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        v += s_f[w][16 * c + r] * *reinterpret_cast<const f32x4_t*>(&red[w][r][(p ^ r) * 4]);
      const int64_t t = row.tok0 + (mr >> a.log2_group);
      if (any)
#pragma unroll 1
        for (int e = 0; e < 4; ++e)
          v[e] += bad_values<D, B>(s_bad, a.mask + t * a.words, a.words, row, a, kvh, 4 * p + e);
      if (row.n_split == 1) {
        const uint2 w = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        *reinterpret_cast<uint2*>(a.out + (t * a.hq + kvh * G + (mr & (G - 1))) * D + 4 * p) = w;
      } else {
        *reinterpret_cast<f32x4_t*>(a.part_o + (part0 + mr) * D + 4 * p) = v;
      }
    }
  }
}

// Merge of split key ranges: with O_s and L_s, a piece's normalised output and
// the log2 of its weights' sum, the row's output is
//     sum_s 2^(L_s - max L) O_s / sum_s 2^(L_s - max L).
// A row (node, q head) takes D / 4 threads of 4 features; with many splits
// several such slots share it, each taking every P-th split, and meet in LDS.
template <int D, class Rows>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(const Rows rows,
                                                              const AttnArgs a) {
  constexpr int DQ = D / 4, SLOTS = kThreads / DQ, U = 8;
  __shared__ float4 s_acc[SLOTS][DQ];
  __shared__ float s_m[SLOTS], s_w[SLOTS];
  const TreeRow row = row_of(rows, blockIdx.x);
  const int per = merge_rows(D, row.n_split);
  const int slot = threadIdx.x / DQ, dq = threadIdx.x % DQ;
  const int P = SLOTS / per, p = slot / per;
  const int x = ((int)blockIdx.x - row.item0) * per + slot % per;  // node * hq + head
  const bool in = x < row.n * a.hq;
  const int node = x / a.hq, h = x % a.hq;
  const int G = 1 << a.log2_group, m_rows = row.n * G;
  const int64_t base = (int64_t)row.part0 +
                       (int64_t)(h >> a.log2_group) * row.n_split * m_rows + node * G +
                       (h & (G - 1));
  float M = -INFINITY, W = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (in) {
    for (int s0 = p; s0 < row.n_split; s0 += P * U) {
      float ls[U];
      float4 o[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {  // past the last split: it again, weight 0
        const int s = s0 + u * P;
        const int64_t pr = base + (int64_t)min(s, row.n_split - 1) * m_rows;
        ls[u] = a.part_lse[pr];
        o[u] = *reinterpret_cast<const float4*>(a.part_o + pr * D + dq * 4);
        if (s >= row.n_split) ls[u] = -INFINITY;
      }
      float m = M;
#pragma unroll
      for (int u = 0; u < U; ++u) m = fmaxf(m, ls[u]);
      const float keep = M == -INFINITY ? 0.f : exp2f(M - m);
      M = m;
      W *= keep;
      acc.x *= keep, acc.y *= keep, acc.z *= keep, acc.w *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (ls[u] == -INFINITY) continue;
        const float w = exp2f(ls[u] - m);
        W += w;
        acc.x += w * o[u].x;
        acc.y += w * o[u].y;
        acc.z += w * o[u].z;
        acc.w += w * o[u].w;
      }
    }
  }
  if (P > 1) {  // uniform
    s_acc[slot][dq] = acc;
    if (dq == 0) s_m[slot] = M, s_w[slot] = W;
    __syncthreads();
    if (p > 0) return;
    for (int k = 1; k < P; ++k) M = fmaxf(M, s_m[k * per + slot]);
    W = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < P; ++k) {
      const float wk = s_w[k * per + slot];
      if (wk == 0.f) continue;
      const float w = exp2f(s_m[k * per + slot] - M);
      const float4 v = s_acc[k * per + slot][dq];
      W += w * wk;
      acc.x += w * v.x;
      acc.y += w * v.y;
      acc.z += w * v.z;
      acc.w += w * v.w;
    }
  }
  if (!in) return;
  const float inv = W == 0.f ? 0.f : 1.f / W;
  uint2 w2;
  w2.x = pack_bf16x2(acc.x * inv, acc.y * inv);
  w2.y = pack_bf16x2(acc.z * inv, acc.w * inv);
  *reinterpret_cast<uint2*>(a.out + ((int64_t)(row.tok0 + node) * a.hq + h) * D + dq * 4) = w2;
}

template <int D, int B>
hipError_t launch_narrow_t(int most, const AttnArgs& a, const TreeRows& rows, int n_rows, int items,
                           hipStream_t s) {
  static_assert(kNarrowRows == 32, "columns");
  return by_size(rows, n_rows, [&](const auto& r) {
    // one column of rows saves registers and products: a request of 16 rows after
    // 300 keys 7.0 us, with two columns 7.9; 32 of them after 1,000 keys 37.4 / 37.8
    if (most <= 16)
      hipLaunchKernelGGL((narrow_kernel<D, B, 1>), dim3(items), dim3(kThreads), 0, s, r, a, a.q,
                         a.k_cache, a.v_cache, a.bt, a.mask);
    else
      hipLaunchKernelGGL((narrow_kernel<D, B, 2>), dim3(items), dim3(kThreads), 0, s, r, a, a.q,
                         a.k_cache, a.v_cache, a.bt, a.mask);
  });
}

}  // namespace

hipError_t launch_narrow(int d, int block, int most, const AttnArgs& a, const TreeRows& rows,
                         int n_rows, int items, hipStream_t s) {
  auto f = d == 128 ? (block == 16 ? launch_narrow_t<128, 16> : launch_narrow_t<128, 32>)
                    : (block == 16 ? launch_narrow_t<64, 16> : launch_narrow_t<64, 32>);
  return f(most, a, rows, n_rows, items, s);
}

hipError_t launch_tree_merge(int d, const AttnArgs& a, const TreeRows& rows, int n_rows, int items,
                             hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    if (d == 128)
      hipLaunchKernelGGL(tree_merge_kernel<128>, dim3(items), dim3(kThreads), 0, s, r, a);
    else
      hipLaunchKernelGGL(tree_merge_kernel<64>, dim3(items), dim3(kThreads), 0, s, r, a);
  });
}

}  // namespace cptree
