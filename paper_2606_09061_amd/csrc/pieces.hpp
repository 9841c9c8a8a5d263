// How key ranges are cut into pieces: the length with the shortest estimated
// time (host side, no HIP).
#pragma once

#include <algorithm>
#include <cstdint>
#include <vector>

namespace cptree {

constexpr int kCus = 256;         // MI355X
constexpr int kSlots = 2 * kCus;  // workgroups at a time: two on each CU

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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

inline Load load_of(const Work& w, uint32_t piece) {
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
inline double time_of(const Load& l, const Cost& c) {
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
inline int best_piece(const Work& w, const Cost& c, double* time) {
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

}  // namespace cptree
