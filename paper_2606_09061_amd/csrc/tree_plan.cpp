// Plan of cp_tree_attn: the kernel, the key ranges' pieces and the workspace.
#include "tree_plan.hpp"

#include <algorithm>

namespace cptree {

namespace {

constexpr int kCus = 256;         // MI355X
constexpr int kSlots = 2 * kCus;  // workgroups at a time: two on each CU

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Estimated times of a kernel, in us: a turn of `turn` keys while every slot
// is busy, and with a CU to itself (bound by the memory's latency); a
// workgroup's start and end; the merge launch and its 1,000 partial rows; and
// the batch's K and V at the rate they come from memory.
struct Cost {
  int turn;
  double loaded, alone, setup, merge, partial, memory;
};

// What the pieces of a kernel are cut from: a row's turns, its workgroups per
// piece and its partial rows per split.
struct Work {
  std::vector<uint32_t> turns, per_split, partial;

  // workgroups, for pieces of `piece` turns
  int64_t workgroups(uint32_t piece) const {
    int64_t n = 0;
    for (size_t i = 0; i < turns.size(); ++i)
      n += (int64_t)((turns[i] + piece - 1) / piece) * per_split[i];
    return n;
  }
};

struct Load {
  int64_t n, work, partial;  // workgroups, their turns, partial rows
  int longest;               // turns of the longest piece
};

Load load_of(const Work& w, uint32_t piece) {
  Load l{0, 0, 0, 0};
  uint32_t longest = 0;
  for (size_t i = 0; i < w.turns.size(); ++i) {
    const uint32_t turns = w.turns[i], s = (turns + piece - 1) / piece;
    l.n += (int64_t)s * w.per_split[i];
    l.work += (int64_t)turns * w.per_split[i];
    longest = std::max(longest, std::min(turns, piece));
    if (s > 1) l.partial += (int64_t)s * w.partial[i];
  }
  l.longest = (int)longest;
  return l;
}

// The estimated time: the slots' share of the work, but at least the longest
// piece, which is slower where workgroups share a CU; with more workgroups than
// slots (the longest come first) the slots end apart by a part of a piece.
double time_of(const Load& l, const Cost& c) {
  const double merge = l.partial ? c.merge + c.partial * l.partial * 1e-3 : 0.0;
  const double share = l.work * c.loaded / kSlots;
  if (l.n <= kCus)  // (a workgroup per CU does not quite reach the memory's rate)
    return std::max(l.longest * c.alone, 1.06 * c.memory) + c.setup + merge;
  if (l.n <= kSlots)
    return std::max({l.longest * 0.75 * c.loaded, share, c.memory}) + c.setup + merge;
  return std::max(share, c.memory) + l.n * c.setup / kSlots + 0.2 * (l.longest * c.loaded + c.setup) + merge;
}

// The pieces' length in turns: of the whole ranges, their parts, and the
// shortest pieces that fill the CUs, the slots once, twice and so on, the one
// with the shortest estimated time, which is added to `time`.
int best_piece(const Work& w, const Cost& c, double* time) {
  const int least = 256 / c.turn;
  const Load whole = load_of(w, 1u << 30);  // longer than any range
  int best = whole.longest;
  *time = time_of(whole, c);
  const auto look = [&](int piece) {
    if (piece >= whole.longest) return;
    const double t = time_of(load_of(w, piece), c);
    if (t < *time) *time = t, best = piece;
  };
  const int64_t rounds = ceil_div(whole.n, kSlots);
  int hi = whole.longest;  // fits the rounds before
  const auto fill = [&](int64_t workgroups) {
    int lo = least;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (w.workgroups(mid) <= workgroups) hi = mid;
      else lo = mid + 1;
    }
    look(hi);
  };
  if (whole.n < kCus) fill(kCus);
  for (int64_t r = rounds; r < rounds + 4 && hi > least; ++r) fill(r * kSlots);
  // few workgroups whatever the pieces: the shortest are not always best
  if (rounds == 1)
    for (int n = 2; n <= 8; n *= 2)
      if (whole.longest / n >= least) look((int)ceil_div(whole.longest, n));
  return best;
}

}  // namespace

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
