// Plan of cp_tree_attn: which kernel a row goes to, the key ranges' pieces and
// the workspace.
#include "tree_plan.hpp"

#include <algorithm>
#include <climits>

namespace cptree {

namespace {

constexpr int kCus = 256;  // MI355X

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A launch's workgroups run `slots` at a time and take `turn` keys per turn; a
// workgroup costs about `setup` turns besides its keys, and a merge pass
// `merge`.  Pieces are not cut below `least` keys.
struct Cost {
  int slots, turn, least;
  double setup, merge;
};

int64_t workgroups(const std::vector<TreeRow>& rows, const std::vector<int>& per_split,
                   int64_t piece) {
  int64_t n = 0;
  for (size_t i = 0; i < rows.size(); ++i)
    n += per_split[i] * ((rows[i].start + rows[i].n + piece - 1) / piece);
  return n;
}

// The piece length with the shortest estimated time: the shortest pieces that
// fill r rounds of the slots, for a few r, or none cut.
int64_t best_piece(const std::vector<TreeRow>& rows, const std::vector<int>& per_split,
                   const Cost& c) {
  int64_t longest = 0, whole = 0;
  for (size_t i = 0; i < rows.size(); ++i) {
    longest = std::max<int64_t>(longest, rows[i].start + rows[i].n);
    whole += per_split[i];
  }
  longest = ceil_div(longest, c.turn) * c.turn;
  const int64_t r0 = ceil_div(whole, c.slots);
  int64_t best = longest;
  double time = r0 * ((double)longest / c.turn + c.setup);
  for (int64_t r = r0; r < r0 + 3; ++r) {
    int64_t lo = ceil_div(c.least, c.turn), hi = longest / c.turn;  // in turns; hi always fits
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (workgroups(rows, per_split, mid * c.turn) <= r * c.slots) hi = mid;
      else lo = mid + 1;
    }
    const double t = r * (hi + c.setup) + c.merge;
    if (hi * c.turn < longest && t < time) time = t, best = hi * c.turn;
  }
  return std::max<int64_t>(best, c.turn);
}

void cut(TreeLaunch& l, const std::vector<int>& per_split, const Cost& c, int hq, TreePlan& out) {
  if (l.rows.empty()) return;
  const int64_t piece = best_piece(l.rows, per_split, c);
  for (TreeRow& t : l.rows) {
    const int64_t keys = t.start + t.n, n = ceil_div(keys, piece);
    t.split_keys = (int32_t)(ceil_div(ceil_div(keys, n), c.turn) * c.turn);
    t.n_split = (int32_t)ceil_div(keys, t.split_keys);
    if (t.n_split == 1) continue;
    const int64_t rows = (int64_t)t.n_split * t.n * hq;
    if (out.partial_rows + rows > INT_MAX) {  // beyond their index type
      t.n_split = 1;
      t.split_keys = (int32_t)(ceil_div(keys, c.turn) * c.turn);
      continue;
    }
    t.part0 = (int32_t)out.partial_rows;
    out.partial_rows += rows;
    out.merge.push_back(t);
  }
  std::stable_sort(l.rows.begin(), l.rows.end(), [](const TreeRow& a, const TreeRow& b) {
    return std::min(a.split_keys, a.start + a.n) > std::min(b.split_keys, b.start + b.n);
  });
}

}  // namespace

void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out) {
  out.narrow.rows.clear();
  out.wide.rows.clear();
  out.merge.clear();
  out.narrow.most = out.wide.most = 0;
  out.partial_rows = 0;
  const int hq = desc.num_q_heads, hkv = desc.num_kv_heads, group = hq / hkv;
  int32_t tok = 0;
  for (int32_t r = 0; r < n_rows; ++r) {
    const cp_row_meta& m = rows[r];
    if (m.chunk_len <= 0) continue;
    TreeLaunch& l = m.chunk_len * group <= kNarrowRows ? out.narrow : out.wide;
    l.rows.push_back(TreeRow{tok, m.chunk_len, m.chunk_start, m.req_id, 0, 1, 0, 0});
    l.most = std::max(l.most, m.chunk_len * group);
    tok += m.chunk_len;
  }
  thread_local std::vector<int> per_split;
  per_split.assign(out.narrow.rows.size(), hkv);
  cut(out.narrow, per_split, Cost{(out.narrow.most <= 32 ? 2 : 1) * kCus, 128, 256, 1.0, 1.0}, hq,
      out);
  const int waves = wide_waves(out.wide.most), tile = 32 * waves;
  per_split.clear();
  for (const TreeRow& t : out.wide.rows)
    per_split.push_back(hkv * (int)ceil_div((int64_t)t.n * group, tile));
  cut(out.wide, per_split, Cost{(waves == 4 ? 2 : 1) * kCus, 64, 256, 2.0, 3.0}, hq, out);
  out.off_lse = (size_t)out.partial_rows * desc.head_dim * 4;
  out.ws_bytes = std::max<size_t>(256, out.off_lse + (size_t)out.partial_rows * 4);
}

}  // namespace cptree
