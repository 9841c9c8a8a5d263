// Random batches through the plan of the tree attention: every key of every
// (node, head) row is covered once, pieces are whole turns, partial rows and
// the workspace do not overlap, and the launches' workgroups find their rows.
#include <cassert>
#include <cstdio>
#include <random>
#include <vector>

#include "tree_plan.hpp"

using namespace cptree;

int main() {
  std::mt19937 gen(7);
  TreePlan p;
  for (int it = 0; it < 4000; ++it) {
    const int group = 1 << gen() % 4, hkv = 1 + gen() % 9, d = gen() % 2 ? 64 : 128;
    const int n_rows = gen() % (it % 50 == 0 ? 400 : 20), longest = 1 << (3 + gen() % 16);
    std::vector<cp_row_meta> rows;
    int64_t nodes = 0;
    for (int r = 0; r < n_rows; ++r) {
      const int start = gen() % longest, n = gen() % 5 ? gen() % 9 : gen() % 257;
      rows.push_back({r, start, n, start + n});
      nodes += n;
    }
    const cp_attn_desc desc{group * hkv, hkv, d, 16, 1, 1 << 20, 512, 1.f};
    plan_tree(desc, rows.data(), n_rows, p);
    const int turn = p.wide ? 64 : 128;
    int64_t seen = 0, partial = 0;
    size_t merged = 0;
    int most = 0, before = 1 << 30;
    std::vector<char> part(p.partial_rows, 0);
    for (const TreeRow& t : p.rows) {
      const int keys = t.start + t.n;
      most = std::max(most, t.n * group);
      seen += t.n;
      assert(p.wide ? t.n <= kMaxNodes : t.n <= kNarrowNodes);
      assert(t.n >= 1 && t.n_split >= 1 && t.split_keys % turn == 0);
      assert((int64_t)t.split_keys * t.n_split >= keys);
      assert((int64_t)t.split_keys * (t.n_split - 1) < keys);  // no empty piece
      assert(tree_tiles(t.n * group, p.wide) * (p.wide ? kWideRows : kNarrowRows) >= t.n * group);
      const int piece = std::min(t.split_keys, keys);
      assert(piece <= before);  // longest first
      before = piece;
      if (t.n_split == 1) continue;
      ++merged;
      const int64_t rows_of = (int64_t)t.n_split * t.n * desc.num_q_heads;
      partial += rows_of;
      for (int64_t i = 0; i < rows_of; ++i) {
        assert(t.part0 + i < p.partial_rows && !part[t.part0 + i]);
        part[t.part0 + i] = 1;
      }
      const int per = merge_rows(d, t.n_split);
      assert(per >= 1 && (1024 / d) % per == 0);
    }
    assert(seen == nodes && most == p.most && partial == p.partial_rows);
    assert(merged == p.merge.size());
    assert(p.off_lse == (size_t)partial * d * 4 && p.off_lse % 16 == 0);
    assert(p.ws_bytes >= p.off_lse + (size_t)partial * 4 && p.ws_bytes >= 256);
  }
  std::puts("ok");
}
