// How the plans of libcpcache are cut into launches (host side, no HIP).
//
// A grid has fewer than 2^32 threads.
#pragma once

#include <limits.h>

#include <algorithm>
#include <vector>

#include "cache_plan.hpp"

namespace cpcache {

// Workgroups that a launch takes at most.
constexpr int64_t max_items(int threads) { return (1ll << 32) / threads - 1; }
static_assert(kMaxItems == max_items(256), "most kernels have 256 threads");

// f(rows of one launch, their number, its items) for rows in batches; the places
// behind them are no item's.  items_of(row) is the number of a row's items, of which
// a launch takes `most`, or a single row's; `item0` is the member that gets those of
// the rows before.
template <class R, int N, class Items, class F>
int by_rows(const std::vector<R>& rows, int32_t R::*item0, int64_t most, Items&& items_of, F&& f) {
  for (size_t r = 0; r < rows.size();) {
    RowsOf<R, N> batch;
    int64_t items = 0;
    int n = 0;
    for (; r < rows.size() && n < N; ++r) {
      const int64_t more = items_of(rows[r]);
      if (n > 0 && items + more > most) break;
      batch.r[n] = rows[r];
      batch.r[n++].*item0 = (int32_t)items;
      items += more;
    }
    for (int i = n; i < N; ++i) batch.r[i] = R{}, batch.r[i].*item0 = INT_MAX;
    const int rc = f(batch, n, (int)items);
    if (rc != CP_OK) return rc;
  }
  return CP_OK;
}

// The launches of cp_page_select: score(rows, their number, workgroups), if any, and
// then choose(the same), or choose alone where one launch does both.
template <class Score, class Choose>
int select_launches(const cp_attn_desc& d, const SelectPlan& p, Score&& score, Choose&& choose) {
  const int64_t hkv = d.num_kv_heads;
  if (p.one == One::kNo) {
    thread_local std::vector<SelectRow> scored;
    scored.clear();
    for (const SelectRow& r : p.rows)
      if (r.stride > 0) scored.push_back(r);
    const int rc = by_rows<SelectRow, kSelectRows>(
        scored, &SelectRow::item0, kMaxItems,
        [&](const SelectRow& r) { return r.n * hkv * ((r.stride + p.chunk - 1) / p.chunk); }, score);
    if (rc != CP_OK) return rc;
  }
  return by_rows<SelectRow, kSelectRows>(
      p.rows, &SelectRow::item0, max_items(p.threads()),
      [&](const SelectRow& r) { return r.n * hkv; }, choose);
}

// A launch of the attention calls, and the merge behind it.
struct AttnLaunch {
  AttnBatch b;
  int n = 0, n_groups = 0;         // its rows and groups
  int items = 0, group_items = 0;  // (tokens, kv head, piece) items of rows, workgroups of groups
  int n_tokens = 0;
  int most = 1;                    // pieces of a row
  int64_t part0 = 0;               // the partial rows of the first item of rows
  bool wide = false, merge = false;
};

// f(launch) for each of a plan's: some of the rows, and the groups that begin among them.
template <class F>
int attn_launches(const cp_attn_desc& d, const AttnPlan& p, F&& f) {
  const int hkv = d.num_kv_heads, G = d.num_q_heads / hkv;
  int64_t part0 = p.row_part0;
  int begun = 0;  // groups whose workgroups have been launched
  for (size_t r = 0; r < p.rows.size();) {
    AttnLaunch x;
    int64_t items = 0, group_items = 0;
    int last = -1;
    x.part0 = part0;
    const int32_t tok0 = p.rows[r].tok0;
    for (; r < p.rows.size() && x.n < kAttnRows; ++r) {
      const TokenRow& t = p.rows[r];
      const int64_t more = (int64_t)t.n_split * p.items_of(t.n) * hkv;
      const bool other = t.group >= 0 && t.group != last, fresh = other && t.group == begun;
      const int64_t shared = fresh ? prefix_items(p.prefix[t.group], G, hkv) : 0;
      if (x.n > 0 && items + group_items + more + shared > kMaxItems) break;
      if (x.n > 0 && merge_items(d, t.tok0 + t.n - tok0, 1) > kMaxItems) break;
      if (other) {
        if (x.n_groups == kGroups) break;
        x.b.g[x.n_groups] = p.prefix[t.group];
        x.b.g[x.n_groups].row0 = x.n;
        // (of a group that began in an earlier launch: no item, it is this one's first)
        x.b.g[x.n_groups++].item0 = (int32_t)group_items;
        x.wide |= fresh && p.prefix[t.group].wide != kNarrow;
        group_items += shared;
        last = t.group;
        if (fresh) ++begun;
      }
      if (t.group >= 0) x.b.g[x.n_groups - 1].row1 = x.n + 1;
      x.b.r[x.n++] = AttnRow{(int32_t)items, t.tok0, t.start, t.req};
      items += more;
      const int pieces = t.n_split + (t.group >= 0 ? p.prefix[t.group].n_split : 0);
      x.merge |= t.n_split > 1 || t.group >= 0;
      x.most = std::max(x.most, pieces);
    }
    const int32_t end = p.rows[r - 1].tok0 + p.rows[r - 1].n;
    for (int i = x.n_groups; i < kGroups; ++i) x.b.g[i] = PrefixRow{}, x.b.g[i].item0 = INT_MAX;
    for (int i = x.n; i <= kAttnRows; ++i) x.b.r[i] = AttnRow{INT_MAX, end, 0, 0};
    x.items = (int)items, x.group_items = (int)group_items, x.n_tokens = end - tok0;
    const int rc = f(x);
    if (rc != CP_OK) return rc;
    if (p.parts) part0 += (items * G) << p.log2_tokens;
  }
  return CP_OK;
}

}  // namespace cpcache
