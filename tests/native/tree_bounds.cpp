// The plan of the tree attention at the ends of its ranges, under UBSan: the
// longest contexts, the most heads and nodes, many rows.  Every key is covered
// once by pieces that the kernels' 32-bit arithmetic can name, and what the
// plan leaves unchecked stays below the bounds that tree_plan.hpp states.
#include <cassert>
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "tree_plan.hpp"

using namespace cptree;

static void check(const cp_attn_desc& desc, const std::vector<cp_row_meta>& rows) {
  static TreePlan p;
  plan_tree(desc, rows.data(), (int32_t)rows.size(), p);
  const int group = desc.num_q_heads / desc.num_kv_heads;
  int64_t partial = 0, cut = 0;
  for (const TreeRow& t : p.rows) {
    const int64_t keys = (int64_t)t.start + t.n, split = t.split_keys;
    assert(split > 0 && t.n_split >= 1);
    assert(split * t.n_split >= keys && split * (t.n_split - 1) < keys);
    assert(split * (t.n_split - 1) + split <= INT32_MAX);  // the last piece's end, as kernels add it
    assert(keys + 255 <= INT32_MAX);                       // and rounded up to turns
    if (t.n_split > 1) partial += (int64_t)t.n_split * t.n * desc.num_q_heads;
    const int64_t items = (int64_t)t.n_split * desc.num_kv_heads * tree_tiles(t.n * group, p.wide);
    if (t.n_split > 1) cut += items;
    else assert(items <= kMaxRowItems);
  }
  assert(partial == p.partial_rows && partial <= kMaxPartialRows);
  assert(cut <= kMaxSplitItems);
}

int main() {
  std::mt19937 gen(3);
  const int heads[][2] = {{1, 1}, {32, 8}, {64, 8}, {8, 1}, {1024, 1024}, {8192, 1024}};
  for (const auto& h : heads)
    for (int d : {64, 128}) {
      const cp_attn_desc desc{h[0], h[1], d, 16, 1, INT32_MAX / 16, 1 << 20, 1.f};
      for (int n : {1, 3, 31, 64, 65, 255, 256})
        for (int ctx : {n, 4096, 1 << 20, 1 << 29, (1 << 30) - 1, 1 << 30})
          for (int copies : {1, 2, 40}) {
            std::vector<cp_row_meta> rows;
            for (int r = 0; r < copies; ++r) rows.push_back({r, ctx - n, n, ctx});
            check(desc, rows);
            // beside short rows, and one longer than the others
            for (int r = 0; r < 200; ++r) {
              const int m = 1 + gen() % (r % 8 ? 9 : 256), c = gen() % 3000;
              rows.push_back({copies + r, c, m, c + m});
            }
            check(desc, rows);
          }
    }
  std::puts("ok");
}
