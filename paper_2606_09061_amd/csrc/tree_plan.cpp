// Plan of cp_tree_attn: the kernel, the key ranges' pieces and the workspace.
#include "tree_plan.hpp"

#include <algorithm>

#include "pieces.hpp"

namespace cptree {

void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out) {
  out.rows.clear();
  out.merge.clear();
  out.most = 0;
  out.partial_rows = 0;
  const int hq = desc.num_q_heads, hkv = desc.num_kv_heads, group = hq / hkv;
  int32_t tok = 0, nodes = 0;
  double keys = 0, read = 0;  // all keys, and as every narrow tile reads them
  for (int32_t r = 0; r < n_rows; ++r) {
    const cp_row_meta& m = rows[r];
    if (m.chunk_len <= 0) continue;
    out.rows.push_back(TreeRow{tok, m.chunk_len, m.chunk_start, m.req_id, 0, 1, 0, 0});
    out.most = std::max(out.most, m.chunk_len * group);
    nodes = std::max(nodes, m.chunk_len);
    keys += m.ctx_len;
    read += (double)m.ctx_len * tree_tiles(m.chunk_len * group, false);
    tok += m.chunk_len;
  }
  out.off_lse = 0;
  out.ws_bytes = 256;
  if (out.rows.empty()) return;

  // Both kernels' best pieces, where there is a choice: a narrow workgroup
  // starts and ends sooner, a wide one takes four times the rows and reads K and
  // V for all of them.  us, narrow / wide, on 32/8 heads: one request of 128 rows
  // after 250 keys 8.4 / 14.0, after 1,000 12.0 / 15.7; 8 of them 10.3 / 14.0
  // and 22.7 / 21.0; 32 of them 32.7 / 18.2 and 85.6 / 37.6.  Of 234 such batches
  // the choice is more than 5 % behind the faster kernel in 5, by 6 to 14 %.
  thread_local Work work;
  const double d = desc.head_dim / 128.0;
  const double per_key = hkv * desc.head_dim * 4.0 / 5.3e6;
  const Cost costs[2] = {{128, 5.5 * d, 0.3 + 1.2 * d, 3.2, 5.5, 0.3 * d, read * per_key},
                         {64, 0.4 + 2.2 * d, 1.0 + 0.2 * d, 7.0, 3.0, 0.2 * d, keys * per_key}};
  int turn = 0, piece = 0;
  double best = 0;
  for (int wide = 0; wide < 2; ++wide) {
    if (wide ? out.most <= kNarrowRows : nodes > kNarrowNodes) continue;
    work.turns.clear(), work.per_split.clear(), work.partial.clear();
    for (const TreeRow& t : out.rows) {
      work.turns.push_back((t.start + t.n + costs[wide].turn - 1) / costs[wide].turn);
      work.per_split.push_back(hkv * tree_tiles(t.n * group, wide));
      work.partial.push_back(t.n * hq);
    }
    double time = 0;
    const int p = best_piece(work, costs[wide], &time);
    if (piece == 0 || time < best) best = time, piece = p, turn = costs[wide].turn, out.wide = wide;
  }
  for (TreeRow& t : out.rows) {
    const int turns = (t.start + t.n + turn - 1) / turn;
    const int n = (turns + piece - 1) / piece, per = (turns + n - 1) / n;
    t.split_keys = per * turn;
    t.n_split = (turns + per - 1) / per;
    if (t.n_split == 1) continue;
    const int64_t partial = (int64_t)t.n_split * t.n * hq;
    t.part0 = (int32_t)out.partial_rows;
    out.partial_rows += partial;
    out.merge.push_back(t);
  }
  std::stable_sort(out.rows.begin(), out.rows.end(), [](const TreeRow& a, const TreeRow& b) {
    return std::min(a.split_keys, a.start + a.n) > std::min(b.split_keys, b.start + b.n);
  });
  out.off_lse = (size_t)out.partial_rows * desc.head_dim * 4;
  out.ws_bytes = std::max<size_t>(256, out.off_lse + (size_t)out.partial_rows * 4);
}

}  // namespace cptree
