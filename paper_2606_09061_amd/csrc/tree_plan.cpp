// Plan of cp_tree_attn: the key ranges' pieces and the workspace.
#include "tree_plan.hpp"

#include <algorithm>

namespace cptree {

namespace {

constexpr int kCus = 256;  // MI355X

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out) {
  out.narrow.clear();
  out.merge.clear();
  out.narrow_rows = 0;
  out.partial_rows = 0;
  const int hq = desc.num_q_heads, hkv = desc.num_kv_heads, group = hq / hkv, d = desc.head_dim;
  int64_t keys = 0, longest = 0;
  for (int32_t r = 0; r < n_rows; ++r)
    if (rows[r].chunk_len > 0) {
      keys += (int64_t)rows[r].ctx_len * hkv;
      longest = std::max<int64_t>(longest, rows[r].ctx_len);
    }
  // Key ranges are cut so that about four workgroups come to a CU, but not
  // below 256 keys, and not at all while none is longer than 512.
  int64_t piece = std::max<int64_t>(2 * kNarrowKeys, ceil_div(keys, 4 * kCus));
  piece = ceil_div(piece, kNarrowKeys) * kNarrowKeys;
  if (longest <= 512) piece = 512;
  int32_t tok = 0;
  for (int32_t r = 0; r < n_rows; ++r) {
    const cp_row_meta& m = rows[r];
    if (m.chunk_len <= 0) continue;
    const int64_t n_split = ceil_div(m.ctx_len, piece);
    const int64_t per = ceil_div(ceil_div(m.ctx_len, n_split), kNarrowKeys) * kNarrowKeys;
    TreeRow t{tok, m.chunk_len, m.chunk_start, m.req_id, 0, (int32_t)ceil_div(m.ctx_len, per),
              (int32_t)per, 0};
    if (t.n_split > 1) {
      t.part0 = (int32_t)out.partial_rows;
      out.partial_rows += (int64_t)t.n_split * m.chunk_len * hq;
      out.merge.push_back(t);
    }
    out.narrow.push_back(t);
    out.narrow_rows = std::max(out.narrow_rows, m.chunk_len * group);
    tok += m.chunk_len;
  }
  out.off_lse = (size_t)out.partial_rows * d * 4;
  out.ws_bytes = std::max<size_t>(256, out.off_lse + (size_t)out.partial_rows * 4);
}

}  // namespace cptree
