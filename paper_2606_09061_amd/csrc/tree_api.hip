// C ABI of libcptree: validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdlib>
#include <new>
#include <vector>

#include "device.hpp"
#include "plan.hpp"
#include "tree_attn.hpp"
#include "tree_ops.hpp"
#include "tree_plan.hpp"

using namespace cptree;

namespace {

// Upper bounds that keep the launches' grids and index types in range.
constexpr int kMaxKvHeads = 1024;
constexpr int64_t kMaxTokens = 1 << 23;
constexpr int32_t kMaxVocab = 1 << 30;
static_assert(kMaxRowItems >= kMaxKvHeads * tree_tiles(8 * kMaxNodes, true) &&
              kMaxRowItems >= kMaxKvHeads * tree_tiles(8 * kNarrowNodes, false));

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool debug_mode() {
  const char* s = std::getenv("CP_DEBUG");
  return s && s[0] == '1';
}

// After a launch; with CP_DEBUG=1 a kernel's error surfaces here.
int finish(hipError_t e, hipStream_t s) {
  if (e != hipSuccess) return CP_ERR_HIP;
  if (debug_mode() &&
      (hipStreamSynchronize(s) != hipSuccess || hipGetLastError() != hipSuccess))
    return CP_ERR_HIP;
  return CP_OK;
}

// CP_DEBUG=1: waits for the stream and checks entries [first, last) of a
// request's table row.
int check_entries(const cp_attn_desc* d, const int32_t* bt, int32_t req, int64_t first,
                  int64_t last, hipStream_t s) {
  if (last <= first) return CP_OK;
  std::vector<int32_t> e(last - first);
  if (hipStreamSynchronize(s) != hipSuccess ||
      hipMemcpy(e.data(), bt + (int64_t)req * d->max_blocks_per_req + first, e.size() * 4,
                hipMemcpyDefault) != hipSuccess)
    return CP_ERR_HIP;
  for (int32_t x : e)
    if (x < 0 || x >= d->num_blocks) return CP_ERR_BAD_META;
  return CP_OK;
}

int check_tables(const cp_attn_desc* d, const int32_t* bt, const cp_row_meta* rows, int32_t n_rows,
                 bool drafted_only, hipStream_t s) {
  if (!debug_mode()) return CP_OK;
  const int64_t B = d->block_size;
  for (int32_t r = 0; r < n_rows; ++r) {
    if (rows[r].chunk_len == 0) continue;
    const int rc = check_entries(d, bt, rows[r].req_id, drafted_only ? rows[r].chunk_start / B : 0,
                                 (rows[r].ctx_len + B - 1) / B, s);
    if (rc != CP_OK) return rc;
  }
  return CP_OK;
}

// Rows without a geometry: the nodes and positions alone.
int check_rows(const cp_row_meta* rows, int32_t n_rows, int most, int64_t* tokens) {
  if (n_rows < 0 || (n_rows > 0 && !rows)) return CP_ERR_INVALID_ARG;
  int64_t total = 0;
  for (int32_t r = 0; r < n_rows; ++r) {
    const cp_row_meta& m = rows[r];
    if (m.chunk_start < 0 || m.chunk_len < 0 || m.chunk_len > most ||
        (int64_t)m.chunk_start + m.chunk_len != m.ctx_len)
      return CP_ERR_BAD_META;
    total += m.chunk_len;
  }
  if (total > kMaxTokens) return CP_ERR_UNSUPPORTED;
  *tokens = total;
  return CP_OK;
}

int check_geometry(const cp_attn_desc* desc, const cp_row_meta* rows, int32_t n_rows, int most,
                   int64_t* tokens) {
  const int rc = cpattn::validate(desc, rows, n_rows);
  if (rc != CP_OK) return rc;
  if (desc->num_kv_heads > kMaxKvHeads) return CP_ERR_UNSUPPORTED;
  return check_rows(rows, n_rows, most, tokens);
}

// Rows that the plan of the attention can take.
int check_attn(const cp_attn_desc* desc, const cp_row_meta* rows, int32_t n_rows, int most,
               int64_t* tokens) {
  const int rc = check_geometry(desc, rows, n_rows, most, tokens);
  if (rc != CP_OK) return rc;
  for (int32_t r = 0; r < n_rows; ++r)
    if (rows[r].chunk_len > 0 && rows[r].ctx_len > CP_TREE_MAX_KEYS) return CP_ERR_UNSUPPORTED;
  return CP_OK;
}

int check_pools(void* const* k_caches, void* const* v_caches, int32_t n_layers) {
  if (n_layers < 0 || (n_layers > 0 && (!k_caches || !v_caches))) return CP_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_layers; ++i)
    if (!k_caches[i] || !v_caches[i] || !aligned(k_caches[i], 16) || !aligned(v_caches[i], 16))
      return CP_ERR_INVALID_ARG;
  return CP_OK;
}

PoolArgs pool_args(const cp_attn_desc* d) {
  return PoolArgs{d->head_dim, d->block_size, d->num_kv_heads, d->max_blocks_per_req,
                  d->num_blocks, 0};
}

int fill_layers(void* const* k_caches, void* const* v_caches, int32_t first, int32_t n_layers,
                Layers& out) {
  const int n = std::min(kLayers, n_layers - first);
  for (int i = 0; i < n; ++i) {
    out.k[i] = static_cast<uint16_t*>(k_caches[first + i]);
    out.v[i] = static_cast<uint16_t*>(v_caches[first + i]);
  }
  return n;
}

// f(rows of one launch, their number, index of the first) for rows in batches.
template <class F>
int by_node_rows(const cp_row_meta* rows, int32_t n_rows, F&& f) {
  int32_t tok = 0;
  for (int32_t r0 = 0; r0 < n_rows; r0 += kNodeRows) {
    NodeRows batch{};
    const int n = std::min(kNodeRows, n_rows - r0);
    for (int i = 0; i < n; ++i) {
      const cp_row_meta& m = rows[r0 + i];
      batch.r[i] = NodeRow{tok, m.chunk_len, m.chunk_start};
      tok += m.chunk_len;
    }
    const int rc = f(batch, n, r0);
    if (rc != CP_OK) return rc;
  }
  return CP_OK;
}

// f(rows of one launch, their number, its workgroups) for rows in batches, the
// places behind them no workgroup's; items_of(row) is the number of a row's
// workgroups.
template <class Items, class F>
int by_tree_rows(const std::vector<TreeRow>& rows, Items&& items_of, F&& f) {
  for (size_t r = 0; r < rows.size();) {
    TreeRows batch;
    int items = 0, n = 0;
    for (; r < rows.size() && n < kTreeRows; ++r) {
      batch.r[n] = rows[r];
      batch.r[n++].item0 = items;
      items += items_of(rows[r]);
    }
    for (int i = n; i < kTreeRows; ++i) batch.r[i] = TreeRow{0, 0, 0, 0, INT_MAX, 1, 0, 0};
    const int rc = f(batch, n, items);
    if (rc != CP_OK) return rc;
  }
  return CP_OK;
}

// One plan per thread, whose vectors keep their capacity.
TreePlan& thread_plan() {
  thread_local TreePlan p;
  return p;
}

int check_forks(const cp_attn_desc* d, const cp_fork* forks, int32_t n_forks) {
  const int64_t cap = (int64_t)d->max_blocks_per_req * d->block_size;
  std::vector<int32_t> src, dst, fresh;
  for (int32_t i = 0; i < n_forks; ++i) {
    const cp_fork& f = forks[i];
    if (f.src_req < 0 || f.src_req >= d->num_reqs_in_table || f.dst_req < 0 ||
        f.dst_req >= d->num_reqs_in_table || f.ctx_len < 0 || f.ctx_len > cap)
      return CP_ERR_BAD_META;
    src.push_back(f.src_req);
    dst.push_back(f.dst_req);
    if (f.ctx_len % d->block_size == 0) continue;
    if (f.block < 0 || f.block >= d->num_blocks) return CP_ERR_BAD_META;
    fresh.push_back(f.block);
  }
  std::sort(src.begin(), src.end());
  std::sort(dst.begin(), dst.end());
  std::sort(fresh.begin(), fresh.end());
  if (std::adjacent_find(dst.begin(), dst.end()) != dst.end() ||
      std::adjacent_find(fresh.begin(), fresh.end()) != fresh.end())
    return CP_ERR_BAD_META;
  for (int32_t x : dst)
    if (std::binary_search(src.begin(), src.end(), x)) return CP_ERR_BAD_META;
  return CP_OK;
}

// No C++ exception crosses the C interface.
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return CP_ERR_HIP;
  }
}

}  // namespace

extern "C" {

int cp_tree_layout(const int32_t* parents, const cp_row_meta* rows, int32_t n_rows,
                   uint64_t* mask, int32_t mask_words, int32_t* positions, void* stream) {
  if (mask_words < 1 || mask_words > kMaxWords) return CP_ERR_INVALID_ARG;
  int64_t tokens = 0;
  const int rc = check_rows(rows, n_rows, 64 * mask_words, &tokens);
  if (rc != CP_OK || tokens == 0) return rc;
  if (!parents || !mask || !positions || !aligned(parents, 4) || !aligned(mask, 8) ||
      !aligned(positions, 4))
    return CP_ERR_INVALID_ARG;
  (void)hipGetLastError();
  hipStream_t s = (hipStream_t)stream;
  return by_node_rows(rows, n_rows, [&](const NodeRows& batch, int n, int) {
    return finish(launch_layout(parents, batch, n, mask, mask_words, positions, s), s);
  });
}

size_t cp_tree_attn_workspace_bytes(const cp_attn_desc* desc, const cp_row_meta* rows,
                                    int32_t n_rows) {
  size_t bytes = 0;
  const int rc = guarded([&] {
    int64_t tokens = 0;
    const int e = check_attn(desc, rows, n_rows, kMaxNodes, &tokens);
    if (e != CP_OK) return e;
    TreePlan& p = thread_plan();
    plan_tree(*desc, rows, n_rows, p);
    bytes = p.ws_bytes;
    return CP_OK;
  });
  return rc == CP_OK ? bytes : 0;
}

int cp_tree_attn(const cp_attn_desc* desc, const void* q, const void* k_cache,
                 const void* v_cache, const int32_t* block_tables, const uint64_t* mask,
                 int32_t mask_words, const cp_row_meta* rows, int32_t n_rows, void* out, void* ws,
                 size_t ws_bytes, void* stream) {
  return guarded([&] {
    if (mask_words < 1 || mask_words > kMaxWords) return CP_ERR_INVALID_ARG;
    int64_t tokens = 0;
    int rc = check_attn(desc, rows, n_rows, 64 * mask_words, &tokens);
    if (rc != CP_OK || tokens == 0) return rc;
    if (!q || !k_cache || !v_cache || !block_tables || !mask || !out || !ws || !aligned(q, 16) ||
        !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) ||
        !aligned(block_tables, 4) || !aligned(mask, 8) || !aligned(ws, 256))
      return CP_ERR_INVALID_ARG;
    TreePlan& p = thread_plan();
    plan_tree(*desc, rows, n_rows, p);
    if (ws_bytes < p.ws_bytes) return CP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, false, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    const int group = desc->num_q_heads / desc->num_kv_heads;
    const AttnArgs a{static_cast<const uint16_t*>(q),
                     static_cast<const uint16_t*>(k_cache),
                     static_cast<const uint16_t*>(v_cache),
                     block_tables,
                     mask,
                     static_cast<uint16_t*>(out),
                     static_cast<float*>(ws),
                     reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.off_lse),
                     mask_words,
                     desc->num_q_heads,
                     desc->num_kv_heads,
                     desc->max_blocks_per_req,
                     __builtin_ctz(group),
                     desc->sm_scale * cpattn::kLog2e};
    const int d = desc->head_dim;
    rc = by_tree_rows(
        p.rows,
        [&](const TreeRow& t) { return t.n_split * desc->num_kv_heads * tree_tiles(t.n * group, p.wide); },
        [&](const TreeRows& batch, int n, int items) {
          const hipError_t e =
              !p.wide    ? launch_narrow(d, desc->block_size, p.most, a, batch, n, items, s)
              : d == 128 ? launch_wide128(desc->block_size, a, batch, items, s)
                         : launch_wide64(desc->block_size, a, batch, items, s);
          return finish(e, s);
        });
    if (rc != CP_OK) return rc;
    return by_tree_rows(
        p.merge,
        [&](const TreeRow& t) {
          const int per = merge_rows(d, t.n_split);
          return (t.n * desc->num_q_heads + per - 1) / per;
        },
        [&](const TreeRows& batch, int n, int items) {
          return finish(launch_tree_merge(d, a, batch, n, items, s), s);
        });
  });
}

size_t cp_tree_verify_workspace_bytes(int64_t n_tokens, int32_t vocab) {
  if (n_tokens < 0 || n_tokens > kMaxTokens || vocab < 1 || vocab > kMaxVocab) return 0;
  return std::max<size_t>(256, (size_t)verify_candidates(n_tokens, vocab) * 8);
}

int cp_tree_verify(const void* logits, int64_t ld, int32_t vocab, const int32_t* tokens,
                   const int32_t* parents, const cp_row_meta* rows, int32_t n_rows,
                   int32_t max_path, int32_t* target, int32_t* path, int32_t* n_accepted,
                   int32_t* next_token, void* ws, size_t ws_bytes, void* stream) {
  if (vocab < 1 || ld < vocab || max_path < 1 || max_path > kMaxNodes) return CP_ERR_INVALID_ARG;
  if (vocab > kMaxVocab) return CP_ERR_UNSUPPORTED;
  int64_t total = 0;
  const int rc = check_rows(rows, n_rows, kMaxNodes, &total);
  if (rc != CP_OK || n_rows == 0) return rc;
  if (!path || !n_accepted || !next_token || !aligned(path, 4) || !aligned(n_accepted, 4) ||
      !aligned(next_token, 4))
    return CP_ERR_INVALID_ARG;
  if (total > 0) {
    if (!logits || !tokens || !parents || !target || !ws || !aligned(logits, 2) ||
        !aligned(tokens, 4) || !aligned(parents, 4) || !aligned(target, 4) || !aligned(ws, 256))
      return CP_ERR_INVALID_ARG;
    const size_t need = (size_t)total * verify_pieces(total, vocab) * 8;
    if (ws_bytes < std::max<size_t>(256, need)) return CP_ERR_WORKSPACE;
  }
  (void)hipGetLastError();
  hipStream_t s = (hipStream_t)stream;
  const int pieces = verify_pieces(total, vocab);
  uint64_t* best = static_cast<uint64_t*>(ws);
  if (total > 0) {
    const int e = finish(launch_argmax(static_cast<const uint16_t*>(logits), ld, vocab, total,
                                       pieces, best, s), s);
    if (e != CP_OK) return e;
  }
  return by_node_rows(rows, n_rows, [&](const NodeRows& batch, int n, int r0) {
    return finish(launch_walk(best, pieces, tokens, parents, batch, n, r0, max_path, target, path,
                              n_accepted, next_token, s), s);
  });
}

int cp_kv_compact(const cp_attn_desc* desc, void* const* k_caches, void* const* v_caches,
                  int32_t n_layers, const int32_t* block_tables, const cp_row_meta* rows,
                  int32_t n_rows, const int32_t* path, int32_t max_path,
                  const int32_t* n_accepted, void* stream) {
  return guarded([&] {
    if (max_path < 1 || max_path > kMaxNodes) return CP_ERR_INVALID_ARG;
    int64_t tokens = 0;
    int rc = check_geometry(desc, rows, n_rows, kMaxNodes, &tokens);
    if (rc == CP_OK) rc = check_pools(k_caches, v_caches, n_layers);
    if (rc != CP_OK || tokens == 0 || n_layers == 0) return rc;
    if (!block_tables || !path || !n_accepted || !aligned(block_tables, 4) || !aligned(path, 4) ||
        !aligned(n_accepted, 4))
      return CP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, true, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    PoolArgs a = pool_args(desc);
    for (int32_t l0 = 0; l0 < n_layers; l0 += kLayers) {
      Layers layers;
      a.n_layers = fill_layers(k_caches, v_caches, l0, n_layers, layers);
      for (int32_t r = 0; r < n_rows;) {
        MoveRows batch{};
        int n = 0;
        for (; r < n_rows && n < kMoveRows; ++r)
          if (rows[r].chunk_len > 0)
            batch.r[n++] = MoveRow{r, rows[r].chunk_len, rows[r].chunk_start, rows[r].req_id};
        if (n == 0) break;
        rc = finish(launch_compact(a, layers, block_tables, batch, n, path, max_path, n_accepted,
                                   s), s);
        if (rc != CP_OK) return rc;
      }
    }
    return CP_OK;
  });
}

int cp_kv_fork(const cp_attn_desc* desc, void* const* k_caches, void* const* v_caches,
               int32_t n_layers, int32_t* block_tables, const cp_fork* forks, int32_t n_forks,
               void* stream) {
  return guarded([&] {
    int rc = cpattn::validate(desc, nullptr, 0);
    if (rc != CP_OK) return rc;
    if (desc->num_kv_heads > kMaxKvHeads) return CP_ERR_UNSUPPORTED;
    if (n_forks < 0 || (n_forks > 0 && !forks)) return CP_ERR_INVALID_ARG;
    rc = check_pools(k_caches, v_caches, n_layers);
    if (rc == CP_OK) rc = check_forks(desc, forks, n_forks);
    if (rc != CP_OK || n_forks == 0) return rc;
    if (!block_tables || !aligned(block_tables, 4)) return CP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    if (debug_mode())
      for (int32_t i = 0; i < n_forks; ++i) {
        rc = check_entries(desc, block_tables, forks[i].src_req, 0,
                           ((int64_t)forks[i].ctx_len + desc->block_size - 1) / desc->block_size,
                           s);
        if (rc != CP_OK) return rc;
      }
    (void)hipGetLastError();
    PoolArgs a = pool_args(desc);
    int32_t l0 = 0;
    do {
      Layers layers;
      a.n_layers = fill_layers(k_caches, v_caches, l0, n_layers, layers);
      for (int32_t i = 0; i < n_forks; i += kForks) {
        Forks batch{};
        const int n = std::min(kForks, n_forks - i);
        std::copy(forks + i, forks + i + n, batch.r);
        rc = finish(launch_fork(a, layers, block_tables, batch, n, l0 == 0, s), s);
        if (rc != CP_OK) return rc;
      }
      l0 += kLayers;
    } while (l0 < n_layers);
    return CP_OK;
  });
}

}  // extern "C"
