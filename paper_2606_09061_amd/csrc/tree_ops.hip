// The calls around the tree attention: layout of drafted trees, greedy
// verification of their logits, compaction of the accepted nodes' K/V and
// forks of requests (include/cp_tree.h).
#include "tree_ops.hpp"

#include <algorithm>

#include "device.hpp"

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
__global__ __launch_bounds__(kThreads) void layout_kernel(const int32_t* __restrict__ parents,
                                                          const NodeRows rows,
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
  uint64_t top = 0;
  auto take = [&](int i) {
    top = max(top, candidate(__uint_as_float((uint32_t)row[i] << 16), i));
  };
  if (piece == 0 && tid < 8 && tid < 8 * w0 - off && tid < vocab) take(tid);
  if (piece == pieces - 1 && tid >= 8 && tid < 16) {
    const int64_t i = (int64_t)8 * w1 - off + tid - 8;
    if (i < vocab) take((int)i);
  }
  for (int w = a + tid; w < b; w += kThreads) {
    const u32x4_t x =
        __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(words + (int64_t)8 * w));
    const int i = 8 * w - off;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      top = max(top, candidate(bf16lo(x[e]), i + 2 * e));
      top = max(top, candidate(bf16hi(x[e]), i + 2 * e + 1));
    }
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
__global__ __launch_bounds__(kThreads) void walk_kernel(
    const uint64_t* __restrict__ best, int pieces, const int32_t* __restrict__ tokens,
    const int32_t* __restrict__ parents, const NodeRows rows, int row0, int max_path,
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

// One workgroup per (row, kv head, layer).  A path rises strictly, so node i's
// source slot is never before its destination: passes of kMoveTokens nodes,
// each read whole before it is written, never overwrite a later pass's
// sources.
template <int D, int B>
__global__ __launch_bounds__(kThreads) void compact_kernel(const Layers layers,
                                                           const MoveRows rows,
                                                           const int32_t* __restrict__ bt, int mbr,
                                                           int num_blocks, int hkv,
                                                           const int32_t* __restrict__ path,
                                                           int max_path,
                                                           const int32_t* __restrict__ n_accepted) {
  constexpr int CH = D / 8;  // 16-byte pieces of a K row
  constexpr int KP = kMoveTokens * CH / kThreads > 0 ? kMoveTokens * CH / kThreads : 1;
  constexpr int VP = kMoveTokens * D / kThreads;
  const MoveRow row = rows.r[blockIdx.x];
  const int h = blockIdx.y, tid = threadIdx.x;
  uint16_t* kc = layers.k[blockIdx.z];
  uint16_t* vc = layers.v[blockIdx.z];
  __shared__ int s_count;
  __shared__ int64_t s_src[kMaxNodes], s_dst[kMaxNodes];  // block * B + slot, -1: no move
  if (tid == 0) s_count = min(min(max(n_accepted[row.row], 0), max_path), row.n);
  __syncthreads();
  const int most = s_count;
  __syncthreads();
  int p = -1;
  if (tid < most) {
    const int32_t* e = path + (int64_t)row.row * max_path + tid;
    p = e[0];
    if (p < 0 || p >= row.n || (tid > 0 && p <= e[-1])) atomicMin(&s_count, tid);
  }
  __syncthreads();
  const int count = s_count;
  if (tid < count) {
    const int src = row.start + p, dst = row.start + tid;
    const int32_t* e = bt + (int64_t)row.req * mbr;
    const int sb = e[src / B], db = e[dst / B];
    const bool ok = src != dst && (unsigned)sb < (unsigned)num_blocks &&
                    (unsigned)db < (unsigned)num_blocks;
    s_src[tid] = ok ? (int64_t)sb * B + src % B : -1;
    s_dst[tid] = ok ? (int64_t)db * B + dst % B : -1;
  }
  __syncthreads();
  for (int i0 = 0; i0 < count; i0 += kMoveTokens) {
    u32x4_t kv[KP];
    uint16_t vv[VP];
#pragma unroll
    for (int x = 0; x < KP; ++x) {
      const int i = i0 + (x * kThreads + tid) / CH;
      if (i < min(count, i0 + kMoveTokens) && s_src[i] >= 0) {
        const int64_t at = ((s_src[i] / B * hkv + h) * B + s_src[i] % B) * D;
        kv[x] = *reinterpret_cast<const u32x4_t*>(kc + at + tid % CH * 8);
      }
    }
#pragma unroll
    for (int x = 0; x < VP; ++x) {
      const int i = i0 + (x * kThreads + tid) / D;
      if (i < count && s_src[i] >= 0)
        vv[x] = vc[((s_src[i] / B * hkv + h) * D + tid % D) * B + s_src[i] % B];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < KP; ++x) {
      const int i = i0 + (x * kThreads + tid) / CH;
      if (i < min(count, i0 + kMoveTokens) && s_dst[i] >= 0) {
        const int64_t at = ((s_dst[i] / B * hkv + h) * B + s_dst[i] % B) * D;
        *reinterpret_cast<u32x4_t*>(kc + at + tid % CH * 8) = kv[x];
      }
    }
#pragma unroll
    for (int x = 0; x < VP; ++x) {
      const int i = i0 + (x * kThreads + tid) / D;
      if (i < count && s_dst[i] >= 0)
        vc[((s_dst[i] / B * hkv + h) * D + tid % D) * B + s_dst[i] % B] = vv[x];
    }
    __syncthreads();
  }
}

constexpr int kForkWords = 4;  // 16-byte words per thread of a page's copy

// Workgroup (x, y, z): piece x of K or V page z in layer y; y == n_layers is
// the fork's table row.
__global__ __launch_bounds__(kThreads) void fork_kernel(const Layers layers, int n_layers,
                                                        const Forks forks, int32_t* bt, int mbr,
                                                        int num_blocks, int block, int page16) {
  const cp_fork f = forks.f[blockIdx.z];
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
  hipLaunchKernelGGL(layout_kernel, dim3(n_rows), dim3(kThreads), 0, s, parents, rows, mask, words,
                     positions);
  return hipGetLastError();
}

int verify_pieces(int64_t n_tokens, int32_t vocab) {
  // about 2,048 workgroups (8 per CU), each of at least four words per thread
  const int64_t want = (2048 + n_tokens - 1) / std::max<int64_t>(n_tokens, 1);
  const int64_t most = std::max<int64_t>(vocab / (4 * 8 * kThreads), 1);
  return (int)std::max<int64_t>(std::min(want, most), 1);
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
  hipLaunchKernelGGL(walk_kernel, dim3(n_rows), dim3(kThreads), 0, s, best, pieces, tokens,
                     parents, rows, row0, max_path, target, path, n_accepted, next_token);
  return hipGetLastError();
}

hipError_t launch_compact(const PoolArgs& a, const Layers& layers, const int32_t* bt,
                          const MoveRows& rows, int n_rows, const int32_t* path, int max_path,
                          const int32_t* n_accepted, hipStream_t s) {
  auto kern = a.d == 128 ? (a.block == 16 ? compact_kernel<128, 16> : compact_kernel<128, 32>)
                         : (a.block == 16 ? compact_kernel<64, 16> : compact_kernel<64, 32>);
  hipLaunchKernelGGL(kern, dim3(n_rows, a.hkv, a.n_layers), dim3(kThreads), 0, s, layers, rows, bt,
                     a.mbr, a.num_blocks, a.hkv, path, max_path, n_accepted);
  return hipGetLastError();
}

hipError_t launch_fork(const PoolArgs& a, const Layers& layers, int32_t* bt, const Forks& forks,
                       int n_forks, bool tables, hipStream_t s) {
  const int page16 = a.hkv * a.d * a.block / 8;
  const int pieces = (page16 + kForkWords * kThreads - 1) / (kForkWords * kThreads);
  hipLaunchKernelGGL(fork_kernel, dim3(2 * pieces, a.n_layers + (tables ? 1 : 0), n_forks),
                     dim3(kThreads), 0, s, layers, a.n_layers, forks, bt, a.mbr, a.num_blocks,
                     a.block, page16);
  return hipGetLastError();
}

}  // namespace cptree
