// The calls around the tree attention: layout of drafted trees, greedy
// verification of their logits, compaction of the accepted nodes' K/V and
// forks of requests (include/cp_tree.h).
#include "tree_ops.hpp"

#include <algorithm>

#include "tree_device.hpp"

namespace cptree {

using cpattn::bf16hi;
using cpattn::bf16lo;
using cpattn::u32x4_t;

namespace {

constexpr int kThreads = 256;
static_assert(kThreads == kMaxNodes, "one thread per node");

// A row's parents in LDS: an index before the node's own, or -1.
__device__ __forceinline__ int load_parent(const int32_t* __restrict__ parents, int tok0, int n,
                                           int j) {
  if (j >= n) return -1;
  const int p = parents[tok0 + j];
  return p >= 0 && p < j ? p : -1;
}

// One workgroup per row, one thread per node, which walks its own chain of
// ancestors in LDS.
template <class Rows>
__global__ __launch_bounds__(kThreads) void layout_kernel(const int32_t* __restrict__ parents,
                                                          const Rows rows,
                                                          uint64_t* __restrict__ mask, int words,
                                                          int32_t* __restrict__ positions) {
  __shared__ int par[kMaxNodes];
  const NodeRow row = rows.r[blockIdx.x];
  const int j = threadIdx.x;
  par[j] = load_parent(parents, row.tok0, row.n, j);
  __syncthreads();
  if (j >= row.n) return;
  uint64_t m[kMaxWords] = {};
  int depth = -1;
  for (int k = j; k >= 0; k = par[k]) {  // falls at every step
#pragma unroll
    for (int w = 0; w < kMaxWords; ++w)
      if (k >> 6 == w) m[w] |= 1ull << (k & 63);
    ++depth;
  }
  const int64_t t = row.tok0 + j;
#pragma unroll
  for (int w = 0; w < kMaxWords; ++w)
    if (w < words) mask[t * words + w] = m[w];
  positions[t] = row.start + depth;
}

// A candidate of the argmax as one number: larger values win, then lower
// indexes.  NaN is above every number; -0 becomes +0.
__device__ __forceinline__ uint64_t candidate(float v, int index) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  const uint32_t key = v != v ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)key << 32 | (uint32_t)~index;
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = max(x, (uint64_t)__shfl_xor((unsigned long long)x, m, 64));
  return x;
}

// 16-byte words of a thread on their way at a time (1,024 nodes of 151,936
// logits: two 40.4 us, four 39.1, eight 39.5; 32 nodes 14.4, 14.8, 15.8).
constexpr int kArgmaxWords = 4;

// best[t][piece] = the best candidate of a piece of node t's logits.  Rows may
// start at any bf16: whole 16-byte words are read as such, the ends one value
// at a time.
__global__ __launch_bounds__(kThreads) void argmax_kernel(const uint16_t* __restrict__ logits,
                                                          int64_t ld, int vocab, int pieces,
                                                          uint64_t* __restrict__ best) {
  const int64_t t = blockIdx.x / pieces;
  const int piece = blockIdx.x % pieces;
  const int tid = threadIdx.x;
  const uint16_t* row = logits + t * ld;
  const int off = (int)(((uintptr_t)row >> 1) & 7);  // elements of the first word before the row
  const int w0 = off ? 1 : 0;                        // whole words [w0, w1): elements 8 w - off ..
  const int w1 = max(w0, (int)(((int64_t)vocab + off) >> 3));
  const int per = (w1 - w0 + pieces - 1) / pieces;
  const int a = min(w0 + piece * per, w1), b = min(a + per, w1);
  const uint16_t* words = row - off;
  // The first of the words with this thread's largest value so far, and the
  // largest magnitude: NaN is above 0x7f80 there, and ignored by the maxima.
  float most = -INFINITY;
  u32x4_t best_word = {0, 0, 0, 0};
  int best_at = -1;
  u16x2_t size = {0, 0};
  auto look = [&](const u32x4_t& x, int w) {
    float m = fmaxf(bf16lo(x[0]), bf16hi(x[0]));
#pragma unroll
    for (int e = 1; e < 4; ++e) m = fmaxf(fmaxf(m, bf16lo(x[e])), bf16hi(x[e]));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2_t, x[e] & 0x7fff7fffu));
    if (m > most || best_at < 0) most = m, best_word = x, best_at = w;
  };
  auto load = [&](int w) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(words + (int64_t)8 * w));
  };
  int w = a + tid;
  for (; w + (kArgmaxWords - 1) * kThreads < b; w += kArgmaxWords * kThreads) {
    u32x4_t x[kArgmaxWords];
#pragma unroll
    for (int u = 0; u < kArgmaxWords; ++u) x[u] = load(w + u * kThreads);
#pragma unroll
    for (int u = 0; u < kArgmaxWords; ++u) look(x[u], w + u * kThreads);
  }
  for (; w < b; w += kThreads) look(load(w), w);
  uint64_t top = 0;
  auto take_word = [&](const u32x4_t& x, int at) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      top = max(top, candidate(bf16lo(x[e]), 8 * at - off + 2 * e));
      top = max(top, candidate(bf16hi(x[e]), 8 * at - off + 2 * e + 1));
    }
  };
  if (max(size[0], size[1]) > 0x7f80) {
    for (w = a + tid; w < b; w += kThreads) take_word(load(w), w);  // rare: the first NaN
  } else if (best_at >= 0) {
    take_word(best_word, best_at);
  }
  auto take = [&](int i) {
    top = max(top, candidate(__uint_as_float((uint32_t)row[i] << 16), i));
  };
  if (piece == 0 && tid < 8 && tid < 8 * w0 - off && tid < vocab) take(tid);
  if (piece == pieces - 1 && tid >= 8 && tid < 16) {
    const int64_t i = (int64_t)8 * w1 - off + tid - 8;
    if (i < vocab) take((int)i);
  }
  __shared__ uint64_t part[kThreads / 64];
  top = wave_max64(top);
  if ((tid & 63) == 0) part[tid >> 6] = top;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) top = max(top, part[i]);
    best[blockIdx.x] = top;
  }
}

// One workgroup per row: the nodes' targets from their pieces, each node's
// first child that agrees, and one thread's walk along those.
template <class Rows>
__global__ __launch_bounds__(kThreads) void walk_kernel(
    const uint64_t* __restrict__ best, int pieces, const int32_t* __restrict__ tokens,
    const int32_t* __restrict__ parents, const Rows rows, int row0, int max_path,
    int32_t* __restrict__ target, int32_t* __restrict__ path, int32_t* __restrict__ n_accepted,
    int32_t* __restrict__ next_token) {
  __shared__ unsigned long long top[kMaxNodes];
  __shared__ int child[kMaxNodes];
  const NodeRow row = rows.r[blockIdx.x];
  const int r = row0 + blockIdx.x, j = threadIdx.x;
  top[j] = 0;
  child[j] = kMaxNodes;
  __syncthreads();
  const int64_t first = (int64_t)row.tok0 * pieces;
  for (int x = j; x < row.n * pieces; x += kThreads)
    atomicMax(&top[x / pieces], (unsigned long long)best[first + x]);
  __syncthreads();
  const int p = load_parent(parents, row.tok0, row.n, j);
  if (j < row.n) target[row.tok0 + j] = (int32_t)~(uint32_t)top[j];
  if (p >= 0 && tokens[row.tok0 + j] == (int32_t)~(uint32_t)top[p]) atomicMin(&child[p], j);
  for (int i = j; i < max_path; i += kThreads) path[(int64_t)r * max_path + i] = -1;
  __syncthreads();
  if (j != 0) return;
  int count = 0, last = -1;
  for (int k = 0; k < row.n && count < max_path; k = child[k]) {  // rises at every step
    path[(int64_t)r * max_path + count++] = k;
    last = k;
  }
  n_accepted[r] = count;
  next_token[r] = last < 0 ? -1 : (int32_t)~(uint32_t)top[last];
}

// Accepted nodes per pass of the compaction.
constexpr int kMoveTokens = 16;

// One wave per (row, kv head, layer).  A path rises strictly, so node i's source
// slot is never before its destination: passes of kMoveTokens nodes, each read
// whole before it is written, never overwrite a later pass's sources.
//
// A token's K is one run of memory, but of its V every feature lies on its own,
// B slots of a page side by side: what reads or writes a value of each feature
// touches all of the page's lines, and, 64 lanes in as many pieces, costs the
// address unit a clock per lane.  So pages of V are read and written whole, in
// runs of a kilobyte (lane l of load q holds 8 slots, piece l % PR, of feature
// q 64 / PR + l / PR): the destination's, and each source's once, for sources
// rise as well.  A value moves over by one exchange in its feature's lanes.  36
// layers of 64 requests, 3.8 nodes each, us: values one by one 65, the
// destination's rows whole and the values gathered 65, pages 60 (some 270 MB).
template <int D, int B, class Rows>
__global__ __launch_bounds__(kThreads) void compact_kernel(const Layers layers, const Rows rows,
                                                           int units,
                                                           const int32_t* __restrict__ bt, int mbr,
                                                           int num_blocks, int hkv,
                                                           const int32_t* __restrict__ path,
                                                           int max_path,
                                                           const int32_t* __restrict__ n_accepted) {
  constexpr int CH = D / 8, TPI = 64 / CH, NI = kMoveTokens / TPI;  // K: pieces, tokens a load
  constexpr int PR = B / 8, NQ = D * PR / 64;  // V: pieces of a feature's slots, loads of a page
  static_assert(kMoveTokens <= B, "a pass's destinations lie in two pages at most");
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6));
  if (unit >= units) return;
  const MoveRow row = rows.r[unit / hkv];
  const int h = unit % hkv;
  uint16_t* kc = layers.k[blockIdx.y];
  uint16_t* vc = layers.v[blockIdx.y];
  const int32_t* entries = path + (int64_t)row.row * max_path;
  const int32_t* table = bt + (int64_t)row.req * mbr;
  const int accepted = n_accepted[row.row], bound = min(max_path, row.n);
  struct Page {
    u32x4_t w[NQ];
  };
  auto v_page = [&](int blk) {
    return reinterpret_cast<u32x4_t*>(vc + ((int64_t)blk * hkv + h) * D * B) + lane;
  };
  auto load_page = [&](int blk) {
    Page p;
    const u32x4_t* a = v_page(blk);
#pragma unroll
    for (int q = 0; q < NQ; ++q) p.w[q] = a[64 * q];
    return p;
  };
  int last = -1;
  for (int i0 = 0; i0 < bound; i0 += 64) {
    // lane l's node i0 + l: its source and destination pages, -1 where it does
    // not move, and its source slot
    const int i = i0 + lane;
    const int p = i < bound ? entries[i] : -1;
    int before = __shfl_up(p, 1, 64);
    if (lane == 0) before = last;
    const uint64_t rises = __builtin_amdgcn_ballot_w64(i < min(accepted, bound) && p > before &&
                                                       p < row.n);
    const int count = ~rises ? __builtin_ctzll(~rises) : 64;  // the first that does not ends it
    int from = -1, to = -1;
    if (lane < count && p != i) {
      from = table[(row.start + p) / B], to = table[(row.start + i) / B];
      if ((unsigned)from >= (unsigned)num_blocks || (unsigned)to >= (unsigned)num_blocks)
        from = -1;
    }
    const int slot = (row.start + p) % B;
    const uint64_t moves = __builtin_amdgcn_ballot_w64(from >= 0);
    for (int j0 = 0; j0 < count; j0 += kMoveTokens) {
      const int n = min(kMoveTokens, count - j0);
      if (!(moves >> j0 & ((1ull << n) - 1))) continue;
      // ---- K: CH lanes a token
      u32x4_t k[NI];
      int64_t k_to[NI];
#pragma unroll
      for (int u = 0; u < NI; ++u) {
        const int t = u * TPI + lane / CH, j = min(j0 + t, 63);
        const int f = __shfl(from, j, 64), d = __shfl(to, j, 64), s = __shfl(slot, j, 64);
        k_to[u] = -1;
        if (t < n && f >= 0) {
          k[u] = *reinterpret_cast<const u32x4_t*>(kc + (((int64_t)f * hkv + h) * B + s) * D +
                                                   lane % CH * 8);
          k_to[u] = (((int64_t)d * hkv + h) * B + (row.start + i0 + j) % B) * D + lane % CH * 8;
        }
      }
      // ---- V: the pass's nodes in one destination page, then those in the next
      for (int ja = j0; ja < j0 + n;) {
        const int s0 = (row.start + i0 + ja) % B, len = min(j0 + n - ja, B - s0);
        const uint64_t here = moves >> ja & ((1ull << len) - 1);
        if (here) {
          const int dst = __builtin_amdgcn_readlane(to, ja + __builtin_ctzll(here));
          // the first page that is another: requested with the destination's
          const uint64_t others =
              __builtin_amdgcn_ballot_w64(from >= 0 && from != dst) >> ja & here;
          int held = others ? __builtin_amdgcn_readlane(from, ja + __builtin_ctzll(others)) : dst;
          Page to_page = load_page(dst), from_page = load_page(held);
          for (uint64_t rest = here; rest; rest &= rest - 1) {
            const int t = __builtin_ctzll(rest), d = s0 + t;  // (uniform, as all that chooses here)
            const int src = __builtin_amdgcn_readlane(from, ja + t);
            const int s = __builtin_amdgcn_readlane(slot, ja + t);
            if (src != dst && src != held) from_page = load_page(held = src);
            const int mine = (lane & ~(PR - 1)) | (s / 8);
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
              uint32_t x = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (s % 8 / 2 == e) x = src == dst ? to_page.w[q][e] : from_page.w[q][e];
              x = __shfl(x, mine, 64);
              x = s & 1 ? x >> 16 : x & 0xffffu;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (d % 8 / 2 == e && lane % PR == d / 8)
                  to_page.w[q][e] = d & 1 ? (to_page.w[q][e] & 0xffffu) | x << 16
                                          : (to_page.w[q][e] & 0xffff0000u) | x;
            }
          }
          u32x4_t* a = v_page(dst);
#pragma unroll
          for (int q = 0; q < NQ; ++q) a[64 * q] = to_page.w[q];
        }
        ja += len;
      }
#pragma unroll
      for (int u = 0; u < NI; ++u)
        if (k_to[u] >= 0) *reinterpret_cast<u32x4_t*>(kc + k_to[u]) = k[u];
    }
    if (count < 64) break;
    last = __builtin_amdgcn_readlane(p, 63);
  }
}

constexpr int kForkWords = 4;  // 16-byte words per thread of a page's copy

// Workgroup (x, y, z): piece x of K or V page z in layer y; y == n_layers is
// the fork's table row.
template <class Forks>
__global__ __launch_bounds__(kThreads) void fork_kernel(const Layers layers, int n_layers,
                                                        const Forks forks, int32_t* bt, int mbr,
                                                        int num_blocks, int block, int page16) {
  const cp_fork f = forks.r[blockIdx.z];
  const int full = f.ctx_len / block;
  const bool partial = f.ctx_len % block != 0;
  const int32_t* src = bt + (int64_t)f.src_req * mbr;
  if ((int)blockIdx.y == n_layers) {
    int32_t* dst = bt + (int64_t)f.dst_req * mbr;
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < full; i += gridDim.x * kThreads)
      dst[i] = src[i];
    if (partial && blockIdx.x == 0 && threadIdx.x == 0) dst[full] = f.block;
    return;
  }
  if (!partial) return;
  const int from = src[full];
  if ((unsigned)from >= (unsigned)num_blocks) return;
  const int pieces = gridDim.x / 2;
  uint16_t* pool = (int)blockIdx.x < pieces ? layers.k[blockIdx.y] : layers.v[blockIdx.y];
  const u32x4_t* a = reinterpret_cast<const u32x4_t*>(pool) + (int64_t)from * page16;
  u32x4_t* b = reinterpret_cast<u32x4_t*>(pool) + (int64_t)f.block * page16;
  const int at = blockIdx.x % pieces * kForkWords * kThreads + threadIdx.x;
  u32x4_t x[kForkWords];
#pragma unroll
  for (int i = 0; i < kForkWords; ++i)
    if (at + i * kThreads < page16) x[i] = a[at + i * kThreads];
#pragma unroll
  for (int i = 0; i < kForkWords; ++i)
    if (at + i * kThreads < page16) b[at + i * kThreads] = x[i];
}

}  // namespace

hipError_t launch_layout(const int32_t* parents, const NodeRows& rows, int n_rows, uint64_t* mask,
                         int words, int32_t* positions, hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL(layout_kernel, dim3(n_rows), dim3(kThreads), 0, s, parents, r, mask, words,
                       positions);
  });
}

// about 2,048 workgroups (8 per CU), each of at least four words per thread
// (1,024 nodes of 151,936 logits 39.1 us; of 512 workgroups 42.5, of 8,192 39.8)
static constexpr int64_t kArgmaxGroups = 2048;

static int64_t most_pieces(int32_t vocab) {
  return std::max<int64_t>(vocab / (4 * 8 * kThreads), 1);
}

int verify_pieces(int64_t n_tokens, int32_t vocab) {
  const int64_t want = (kArgmaxGroups + n_tokens - 1) / std::max<int64_t>(n_tokens, 1);
  return (int)std::max<int64_t>(std::min(want, most_pieces(vocab)), 1);
}

// n ceil(2048 / n) falls here and there; 2048 + n - 1, its bound, only rises.
int64_t verify_candidates(int64_t n_tokens, int32_t vocab) {
  return std::min(n_tokens * most_pieces(vocab), n_tokens + kArgmaxGroups - 1);
}

hipError_t launch_argmax(const uint16_t* logits, int64_t ld, int32_t vocab, int64_t n_tokens,
                         int pieces, uint64_t* best, hipStream_t s) {
  hipLaunchKernelGGL(argmax_kernel, dim3((unsigned)(n_tokens * pieces)), dim3(kThreads), 0, s,
                     logits, ld, vocab, pieces, best);
  return hipGetLastError();
}

hipError_t launch_walk(const uint64_t* best, int pieces, const int32_t* tokens,
                       const int32_t* parents, const NodeRows& rows, int n_rows, int row0,
                       int max_path, int32_t* target, int32_t* path, int32_t* n_accepted,
                       int32_t* next_token, hipStream_t s) {
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL(walk_kernel, dim3(n_rows), dim3(kThreads), 0, s, best, pieces, tokens,
                       parents, r, row0, max_path, target, path, n_accepted, next_token);
  });
}

template <int D, int B>
static hipError_t launch_compact_t(const PoolArgs& a, const Layers& layers, const int32_t* bt,
                                   const MoveRows& rows, int n_rows, const int32_t* path,
                                   int max_path, const int32_t* n_accepted, hipStream_t s) {
  const int units = n_rows * a.hkv, waves = kThreads / 64;
  return by_size(rows, n_rows, [&](const auto& r) {
    hipLaunchKernelGGL((compact_kernel<D, B>), dim3((units + waves - 1) / waves, a.n_layers),
                       dim3(kThreads), 0, s, layers, r, units, bt, a.mbr, a.num_blocks, a.hkv,
                       path, max_path, n_accepted);
  });
}

hipError_t launch_compact(const PoolArgs& a, const Layers& layers, const int32_t* bt,
                          const MoveRows& rows, int n_rows, const int32_t* path, int max_path,
                          const int32_t* n_accepted, hipStream_t s) {
  auto f = a.d == 128 ? (a.block == 16 ? launch_compact_t<128, 16> : launch_compact_t<128, 32>)
                      : (a.block == 16 ? launch_compact_t<64, 16> : launch_compact_t<64, 32>);
  return f(a, layers, bt, rows, n_rows, path, max_path, n_accepted, s);
}

hipError_t launch_fork(const PoolArgs& a, const Layers& layers, int32_t* bt, const Forks& forks,
                       int n_forks, bool tables, hipStream_t s) {
  const int page16 = a.hkv * a.d * a.block / 8;
  const int pieces = (page16 + kForkWords * kThreads - 1) / (kForkWords * kThreads);
  return by_size(forks, n_forks, [&](const auto& f) {
    hipLaunchKernelGGL(fork_kernel, dim3(2 * pieces, a.n_layers + (tables ? 1 : 0), n_forks),
                       dim3(kThreads), 0, s, layers, a.n_layers, f, bt, a.mbr, a.num_blocks,
                       a.block, page16);
  });
}

}  // namespace cptree
