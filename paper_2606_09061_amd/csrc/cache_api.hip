// C ABI of libcpcache: validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <vector>

#include "cache_batches.hpp"
#include "cache_kernels.hpp"
#include "device.hpp"
#include "plan.hpp"

using namespace cpcache;

namespace {

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Whether none of the pointers is null or misaligned.
bool usable(size_t a, std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p || !aligned(p, a)) return false;
  return true;
}

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

// Entries [first, last) of a request's table row, behind the stream's work.
int read_entries(const cp_attn_desc* d, const int32_t* bt, int32_t req, int64_t first, int64_t last,
                 hipStream_t s, std::vector<int32_t>& out) {
  out.assign(std::max<int64_t>(0, last - first), 0);
  if (out.empty()) return CP_OK;
  if (hipStreamSynchronize(s) != hipSuccess ||
      hipMemcpy(out.data(), bt + (int64_t)req * d->max_blocks_per_req + first, out.size() * 4,
                hipMemcpyDefault) != hipSuccess)
    return CP_ERR_HIP;
  return CP_OK;
}

// CP_DEBUG=1: the entries that the rows read, or write to, are blocks.
int check_tables(const cp_attn_desc* d, const int32_t* bt, const cp_row_meta* rows, int32_t n_rows,
                 bool written_only, hipStream_t s) {
  if (!debug_mode()) return CP_OK;
  std::vector<int32_t> e;
  const int64_t B = d->block_size;
  for (int32_t r = 0; r < n_rows; ++r) {
    if (rows[r].chunk_len == 0) continue;
    const int rc = read_entries(d, bt, rows[r].req_id, written_only ? rows[r].chunk_start / B : 0,
                                (rows[r].ctx_len + B - 1) / B, s, e);
    if (rc != CP_OK) return rc;
    for (int32_t x : e)
      if (x < 0 || x >= d->num_blocks) return CP_ERR_BAD_META;
  }
  return CP_OK;
}

int check_batch(const cp_attn_desc* desc, const cp_row_meta* rows, int32_t n_rows,
                int64_t* tokens) {
  const int rc = cpattn::validate(desc, rows, n_rows);
  if (rc != CP_OK) return rc;
  if (desc->num_kv_heads > kMaxKvHeads) return CP_ERR_UNSUPPORTED;
  int64_t total = 0;
  for (int32_t r = 0; r < n_rows; ++r) {
    if (rows[r].chunk_len > 0 && rows[r].ctx_len > CP_CACHE_MAX_KEYS) return CP_ERR_UNSUPPORTED;
    total += rows[r].chunk_len;
  }
  if (total > kMaxTokens || total * desc->num_q_heads > kMaxPairs) return CP_ERR_UNSUPPORTED;
  *tokens = total;
  return CP_OK;
}

int check_groups(const cp_row_meta* rows, int32_t n_rows, const cp_prefix_group* groups,
                 int32_t n_groups) {
  if (n_groups < 0 || (n_groups > 0 && !groups)) return CP_ERR_INVALID_ARG;
  int64_t next = 0;
  for (int32_t g = 0; g < n_groups; ++g) {
    const cp_prefix_group& p = groups[g];
    if (p.first_row < next || p.n_rows < 0 || (int64_t)p.first_row + p.n_rows > n_rows ||
        p.common < 0)
      return CP_ERR_BAD_META;
    next = (int64_t)p.first_row + p.n_rows;
    for (int32_t r = p.first_row; r < next; ++r)
      if (rows[r].chunk_len > 0 && p.common > rows[r].chunk_start) return CP_ERR_BAD_META;
  }
  return CP_OK;
}

// CP_DEBUG=1: the table rows of a group name the same blocks for its common keys.
int check_shared(const cp_attn_desc* d, const int32_t* bt, const cp_row_meta* rows,
                 const cp_prefix_group* groups, int32_t n_groups, hipStream_t s) {
  if (!debug_mode()) return CP_OK;
  std::vector<int32_t> first, e;
  for (int32_t g = 0; g < n_groups; ++g) {
    bool any = false;
    for (int32_t r = groups[g].first_row; r < groups[g].first_row + groups[g].n_rows; ++r) {
      if (rows[r].chunk_len == 0) continue;
      const int rc = read_entries(d, bt, rows[r].req_id, 0, groups[g].common / d->block_size, s,
                                  any ? e : first);
      if (rc != CP_OK) return rc;
      if (any && e != first) return CP_ERR_BAD_META;
      any = true;
    }
  }
  return CP_OK;
}

bool pages_in_range(int32_t n_pages) { return n_pages >= 1 && n_pages <= CP_CACHE_MAX_PAGES; }

// One plan per thread, whose vectors keep their capacity.
AttnPlan& thread_plan() {
  thread_local AttnPlan p;
  return p;
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

AttnArgs attn_args(const cp_attn_desc* d, const AttnPlan& p, const void* q, const void* k_cache,
                   const void* v_cache, const int32_t* bt, const int32_t* pages, int32_t n_pages,
                   void* out, void* ws) {
  return AttnArgs{static_cast<const uint16_t*>(q),
                  static_cast<const uint16_t*>(k_cache),
                  static_cast<const uint16_t*>(v_cache),
                  bt,
                  pages,
                  static_cast<uint16_t*>(out),
                  static_cast<float*>(ws),
                  reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.off_lse),
                  d->num_q_heads,
                  d->num_kv_heads,
                  d->max_blocks_per_req,
                  __builtin_ctz(d->num_q_heads / d->num_kv_heads),
                  n_pages,
                  p.piece,
                  0,
                  0,
                  __builtin_ctz(p.unit_waves),
                  p.log2_tokens,
                  0,
                  0,
                  d->sm_scale * cpattn::kLog2e};
}

// The launches of a plan, and the merges of what has several pieces.
int launch_plan(const cp_attn_desc* d, const AttnPlan& p, AttnArgs a, hipStream_t s) {
  const int D = d->head_dim, B = d->block_size;
  return attn_launches(*d, p, [&](const AttnLaunch& x) {
    a.part0 = (int)x.part0, a.n_groups = x.n_groups, a.group_items = x.group_items;
    a.items = x.items;
    const int per = std::max(1, 4 / p.unit_waves), all = x.group_items + (x.items + per - 1) / per;
    const hipError_t e = a.pages    ? launch_pages(D, B, a, x.b, x.n, all, s)
                         : !x.wide  ? launch_shared(D, B, a, x.b, x.n, all, s)
                         : D == 128 ? launch_shared_wide128(B, a, x.b, all, s)
                                    : launch_shared_wide64(B, a, x.b, all, s);
    int rc = finish(e, s);
    if (rc == CP_OK && x.merge)
      rc = finish(launch_cache_merge(*d, a, x.b, x.n, x.n_tokens, x.most, s), s);
    return rc;
  });
}

}  // namespace

extern "C" {

int cp_qkv_append(const cp_attn_desc* desc, const void* qkv, const void* q_norm_w,
                  const void* k_norm_w, const int32_t* positions, double theta, float eps, void* q,
                  void* k_cache, void* v_cache, const int32_t* block_tables,
                  const cp_row_meta* rows, int32_t n_rows, void* stream) {
  return guarded([&] {
    int64_t tokens = 0;
    int rc = check_batch(desc, rows, n_rows, &tokens);
    if (rc != CP_OK) return rc;
    if (!(theta > 1.0) || !std::isfinite(theta) || !(eps > 0.f)) return CP_ERR_INVALID_ARG;
    if (tokens == 0) return CP_OK;
    if (!usable(16, {qkv, q_norm_w, k_norm_w, q, k_cache, v_cache}) || !usable(4, {block_tables}) ||
        !aligned(positions, 4))
      return CP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, true, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    const int D = desc->head_dim, B = desc->block_size;
    const AppendArgs a{static_cast<const uint16_t*>(qkv),
                       static_cast<const uint16_t*>(q_norm_w),
                       static_cast<const uint16_t*>(k_norm_w),
                       positions,
                       static_cast<uint16_t*>(q),
                       static_cast<uint16_t*>(k_cache),
                       static_cast<uint16_t*>(v_cache),
                       block_tables,
                       exp2(-2.0 / D * log2(theta)),
                       exp2(-16.0 / D * log2(theta)),
                       eps,
                       desc->num_q_heads,
                       desc->num_kv_heads,
                       desc->max_blocks_per_req,
                       desc->num_blocks};
    // pieces that end with a page
    thread_local std::vector<AppendRow> pieces;
    pieces.clear();
    int32_t tok = 0;
    for (int32_t r = 0; r < n_rows; ++r) {
      const cp_row_meta& m = rows[r];
      for (int32_t j = 0; j < m.chunk_len;) {
        const int32_t at = m.chunk_start + j;
        const int32_t n = std::min(m.chunk_len - j, kPieceTokens - at % B);
        pieces.push_back(AppendRow{tok + j, 0, n, m.req_id, at, 0});
        j += n;
      }
      tok += m.chunk_len;
    }
    const int per = append_v_items(D, B, desc->num_kv_heads);
    const auto items_of = [&](const AppendRow& p) {
      return (int64_t)((p.start + p.n - 1) / B - p.start / B + 1) * per;
    };
    return by_rows<AppendRow, kAppendRows>(
        pieces, &AppendRow::item0, kMaxItems, items_of,
        [&](AppendRows& batch, int n, int items) {
          int32_t before = 0;
          for (int i = 0; i < n; ++i) {
            batch.r[i].first = before;
            before += batch.r[i].n;
          }
          for (int i = n; i < kAppendRows; ++i) batch.r[i].first = INT_MAX;
          return finish(launch_append(D, B, a, batch, n, before, items, s), s);
        });
  });
}

int cp_page_bounds(const cp_attn_desc* desc, const void* k_cache, const int32_t* block_tables,
                   const cp_row_meta* rows, int32_t n_rows, void* bounds, void* stream) {
  return guarded([&] {
    int64_t tokens = 0;
    int rc = check_batch(desc, rows, n_rows, &tokens);
    if (rc != CP_OK || tokens == 0) return rc;
    if (!usable(16, {k_cache, bounds}) || !usable(4, {block_tables})) return CP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, true, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    const BoundsArgs a{static_cast<const uint16_t*>(k_cache), block_tables,
                       static_cast<uint16_t*>(bounds), desc->num_kv_heads,
                       desc->max_blocks_per_req, desc->num_blocks};
    struct Piece {
      int32_t item0, req, page0, ctx, pages;
    };
    thread_local std::vector<Piece> pieces;
    pieces.clear();
    const int32_t B = desc->block_size;
    for (int32_t r = 0; r < n_rows; ++r) {
      const cp_row_meta& m = rows[r];
      if (m.chunk_len == 0) continue;
      for (int32_t p = m.chunk_start / B, end = (m.ctx_len - 1) / B + 1; p < end; p += kPiecePages)
        pieces.push_back(Piece{0, m.req_id, p, m.ctx_len, std::min(kPiecePages, end - p)});
    }
    return by_rows<Piece, kBoundsRows>(
        pieces, &Piece::item0, kMaxItems / desc->num_kv_heads, [](const Piece& p) { return p.pages; },
        [&](RowsOf<Piece, kBoundsRows>& batch, int n, int pages) {
          BoundsRows r;
          for (int i = 0; i < kBoundsRows; ++i)
            r.r[i] = BoundsRow{batch.r[i].item0, batch.r[i].req, batch.r[i].page0, batch.r[i].ctx};
          return finish(launch_bounds(desc->head_dim, B, a, r, n, pages, s), s);
        });
  });
}

size_t cp_page_select_workspace_bytes(const cp_attn_desc* desc, const cp_row_meta* rows,
                                      int32_t n_rows, int32_t n_pages) {
  size_t bytes = 0;
  const int rc = guarded([&] {
    int64_t tokens = 0;
    const int e = check_batch(desc, rows, n_rows, &tokens);
    if (e != CP_OK) return e;
    if (!pages_in_range(n_pages)) return CP_ERR_INVALID_ARG;
    thread_local SelectPlan plan;
    plan_select(*desc, rows, n_rows, n_pages, plan);
    bytes = std::max<size_t>(256, (size_t)plan.scores * 8);
    return CP_OK;
  });
  return rc == CP_OK ? bytes : 0;
}

int cp_page_select(const cp_attn_desc* desc, const void* q, const void* bounds,
                   const int32_t* block_tables, const cp_row_meta* rows, int32_t n_rows,
                   int32_t n_pages, int32_t n_first, int32_t n_last, int32_t* pages, void* ws,
                   size_t ws_bytes, void* stream) {
  return guarded([&] {
    int64_t tokens = 0;
    int rc = check_batch(desc, rows, n_rows, &tokens);
    if (rc != CP_OK) return rc;
    if (!pages_in_range(n_pages) || n_first < 0 || n_last < 0 ||
        (int64_t)n_first + n_last > n_pages)
      return CP_ERR_INVALID_ARG;
    if (tokens == 0) return CP_OK;
    if (!usable(16, {q, bounds}) || !usable(4, {block_tables, pages}) || !usable(256, {ws}))
      return CP_ERR_INVALID_ARG;
    thread_local SelectPlan plan;
    plan_select(*desc, rows, n_rows, n_pages, plan);
    if (ws_bytes < std::max<size_t>(256, (size_t)plan.scores * 8)) return CP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, false, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    const SelectArgs a{static_cast<const uint16_t*>(q),
                       static_cast<const uint16_t*>(bounds),
                       block_tables,
                       pages,
                       static_cast<uint64_t*>(ws),
                       desc->num_q_heads,
                       desc->num_kv_heads,
                       desc->max_blocks_per_req,
                       desc->num_blocks,
                       desc->block_size,
                       n_pages,
                       n_first,
                       n_last,
                       plan.chunk};
    return select_launches(
        *desc, plan,
        [&](SelectRows& batch, int n, int items) {
          return finish(launch_score(desc->head_dim, a, batch, n, items, s), s);
        },
        [&](SelectRows& batch, int n, int items) {
          return finish(plan.one == One::kNo
                            ? launch_choose(a, batch, n, items, plan.most, s)
                            : launch_select(desc->head_dim, a, batch, n, items, plan.one, s),
                        s);
        });
  });
}

size_t cp_page_attn_workspace_bytes(const cp_attn_desc* desc, const cp_row_meta* rows,
                                    int32_t n_rows, int32_t n_pages) {
  size_t bytes = 0;
  const int rc = guarded([&] {
    int64_t tokens = 0;
    const int e = check_batch(desc, rows, n_rows, &tokens);
    if (e != CP_OK) return e;
    if (!pages_in_range(n_pages)) return CP_ERR_INVALID_ARG;
    AttnPlan& p = thread_plan();
    if (!plan_pages(*desc, rows, n_rows, n_pages, p)) return CP_ERR_UNSUPPORTED;
    bytes = p.ws_bytes;
    return CP_OK;
  });
  return rc == CP_OK ? bytes : 0;
}

int cp_page_attn(const cp_attn_desc* desc, const void* q, const void* k_cache, const void* v_cache,
                 const int32_t* block_tables, const int32_t* pages, int32_t n_pages,
                 const cp_row_meta* rows, int32_t n_rows, void* out, void* ws, size_t ws_bytes,
                 void* stream) {
  return guarded([&] {
    int64_t tokens = 0;
    int rc = check_batch(desc, rows, n_rows, &tokens);
    if (rc != CP_OK) return rc;
    if (!pages_in_range(n_pages)) return CP_ERR_INVALID_ARG;
    if (tokens == 0) return CP_OK;
    if (!usable(16, {q, k_cache, v_cache, out}) || !usable(4, {block_tables, pages}) ||
        !usable(256, {ws}))
      return CP_ERR_INVALID_ARG;
    AttnPlan& p = thread_plan();
    if (!plan_pages(*desc, rows, n_rows, n_pages, p)) return CP_ERR_UNSUPPORTED;
    if (ws_bytes < p.ws_bytes) return CP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, false, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    return launch_plan(desc, p,
                       attn_args(desc, p, q, k_cache, v_cache, block_tables, pages, n_pages, out, ws),
                       s);
  });
}

size_t cp_prefix_attn_workspace_bytes(const cp_attn_desc* desc, const cp_row_meta* rows,
                                      int32_t n_rows, const cp_prefix_group* groups,
                                      int32_t n_groups) {
  size_t bytes = 0;
  const int rc = guarded([&] {
    int64_t tokens = 0;
    int e = check_batch(desc, rows, n_rows, &tokens);
    if (e == CP_OK) e = check_groups(rows, n_rows, groups, n_groups);
    if (e != CP_OK) return e;
    AttnPlan& p = thread_plan();
    if (!plan_prefix(*desc, rows, n_rows, groups, n_groups, p)) return CP_ERR_UNSUPPORTED;
    bytes = p.ws_bytes;
    return CP_OK;
  });
  return rc == CP_OK ? bytes : 0;
}

int cp_prefix_attn(const cp_attn_desc* desc, const void* q, const void* k_cache,
                   const void* v_cache, const int32_t* block_tables, const cp_row_meta* rows,
                   int32_t n_rows, const cp_prefix_group* groups, int32_t n_groups, void* out,
                   void* ws, size_t ws_bytes, void* stream) {
  return guarded([&] {
    int64_t tokens = 0;
    int rc = check_batch(desc, rows, n_rows, &tokens);
    if (rc == CP_OK) rc = check_groups(rows, n_rows, groups, n_groups);
    if (rc != CP_OK || tokens == 0) return rc;
    if (!usable(16, {q, k_cache, v_cache, out}) || !usable(4, {block_tables}) || !usable(256, {ws}))
      return CP_ERR_INVALID_ARG;
    AttnPlan& p = thread_plan();
    if (!plan_prefix(*desc, rows, n_rows, groups, n_groups, p)) return CP_ERR_UNSUPPORTED;
    if (ws_bytes < p.ws_bytes) return CP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    rc = check_tables(desc, block_tables, rows, n_rows, false, s);
    if (rc == CP_OK) rc = check_shared(desc, block_tables, rows, groups, n_groups, s);
    if (rc != CP_OK) return rc;
    (void)hipGetLastError();
    return launch_plan(
        desc, p, attn_args(desc, p, q, k_cache, v_cache, block_tables, nullptr, 0, out, ws), s);
  });
}

}  // extern "C"
