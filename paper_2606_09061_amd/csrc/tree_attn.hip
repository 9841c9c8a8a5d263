// Attention of drafted trees over the paged cache (include/cp_tree.h).
#include "tree_attn.hpp"

#include "device.hpp"

namespace cptree {

using cpattn::bf16hi;
using cpattn::bf16lo;
using cpattn::to_bf16;
using cpattn::wave_max;
using cpattn::wave_sum;

namespace {

constexpr int kThreads = 256;

// One workgroup per (node, q head), 256 keys at a time: a thread scores one
// key, the chunk's weights meet in LDS, and a thread then sums one feature's
// values over half the chunk.  Keys without weight are not multiplied.
template <int D, int B>
__global__ __launch_bounds__(kThreads) void tree_attn_kernel(const TreeRows rows, int n_rows,
                                                             const AttnArgs a) {
  __shared__ float s_q[D], s_p[kThreads], s_red[4], s_o[kThreads];
  const int tid = threadIdx.x, h = blockIdx.y;
  int r = 0;
  while (r + 1 < n_rows && rows.r[r + 1].item0 <= (int)blockIdx.x) ++r;
  const TreeRow row = rows.r[r];
  const int64_t t = row.tok0 + (int)blockIdx.x - row.item0;
  const int kvh = h / (a.hq / a.hkv);
  if (tid < D) s_q[tid] = __uint_as_float((uint32_t)a.q[(t * a.hq + h) * D + tid] << 16);
  __syncthreads();
  const int32_t* bt = a.bt + (int64_t)row.req * a.mbr;
  const int ctx = row.start + row.n, d = tid % D, part = tid / D;
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int k0 = 0; k0 < ctx; k0 += kThreads) {
    const int key = k0 + tid, j = key - row.start;
    bool seen = key < ctx;
    if (seen && j >= 0) seen = (a.mask[t * a.words + (j >> 6)] >> (j & 63)) & 1;
    float s = -INFINITY;
    if (seen) {
      const uint16_t* k =
          a.k_cache + (((int64_t)bt[key / B] * a.hkv + kvh) * B + key % B) * D;
      s = 0.f;
      for (int c = 0; c < D / 8; ++c) {
        const uint4 w = cpattn::ld_global16(k + c * 8);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        for (int e = 0; e < 4; ++e)
          s += bf16lo(x[e]) * s_q[c * 8 + 2 * e] + bf16hi(x[e]) * s_q[c * 8 + 2 * e + 1];
      }
      s *= a.scale_log2;
    }
    const float top = wave_max(s);
    if ((tid & 63) == 0) s_red[tid >> 6] = top;
    __syncthreads();
    const float mn = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float alpha = m == -INFINITY ? 0.f : exp2f(m - mn);
    m = mn;
    s_p[tid] = seen ? exp2f(s - m) : 0.f;
    __syncthreads();
    o *= alpha;
    l *= alpha;
    for (int i = part; i < min(kThreads, ctx - k0); i += kThreads / D) {
      const float p = s_p[i];
      if (p == 0.f) continue;
      l += p;
      const int x = k0 + i;
      const uint16_t v = a.v_cache[(((int64_t)bt[x / B] * a.hkv + kvh) * D + d) * B + x % B];
      o += p * __uint_as_float((uint32_t)v << 16);
    }
    __syncthreads();
  }
  s_o[tid] = o;
  s_p[tid] = l;
  __syncthreads();
  if (tid >= D) return;
  o = 0.f;
  l = 0.f;
  for (int i = tid; i < kThreads; i += D) o += s_o[i], l += s_p[i];
  a.out[(t * a.hq + h) * D + tid] = to_bf16(l == 0.f ? 0.f : o / l);
}

}  // namespace

hipError_t launch_attn(int d, int block, const AttnArgs& a, const TreeRows& rows, int n_rows,
                       int items, hipStream_t s) {
  auto kern = d == 128 ? (block == 16 ? tree_attn_kernel<128, 16> : tree_attn_kernel<128, 32>)
                       : (block == 16 ? tree_attn_kernel<64, 16> : tree_attn_kernel<64, 32>);
  hipLaunchKernelGGL(kern, dim3(items, a.hq), dim3(kThreads), 0, s, rows, n_rows, a);
  return hipGetLastError();
}

}  // namespace cptree
