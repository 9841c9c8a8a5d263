// Random batches through the plans of libcpcache: every token and key range is
// covered once, partial rows do not overlap and fit the workspace, pieces keep to
// their bounds.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "cache_plan.hpp"

using namespace cpcache;

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      fprintf(stderr, "line %d: %s\n", __LINE__, #x);         \
      exit(1);                                                \
    }                                                         \
  } while (0)

namespace {

std::mt19937_64 rng(7);

int64_t uniform(int64_t lo, int64_t hi) {
  return std::uniform_int_distribution<int64_t>(lo, hi)(rng);
}

int32_t spread(int64_t lo, int64_t hi) {  // over the logarithm
  const double a = std::uniform_real_distribution<double>(std::log(lo + 1.0), std::log(hi + 1.0))(rng);
  return (int32_t)std::min<int64_t>(hi, std::max<int64_t>(lo, (int64_t)(std::exp(a) - 1.0)));
}

struct Range {
  int64_t first, n;
};

void no_overlap(std::vector<Range>& r, int64_t total) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.first < b.first; });
  int64_t at = 0;
  for (const Range& x : r) {
    CHECK(x.first >= at);
    at = x.first + x.n;
  }
  CHECK(at <= total);
}

void check(const cp_attn_desc& d, const std::vector<cp_row_meta>& rows,
           const std::vector<cp_prefix_group>& groups, int32_t n_pages) {
  static AttnPlan p;
  const int64_t B = d.block_size, hq = d.num_q_heads, hkv = d.num_kv_heads;
  for (int which = 0; which < 2; ++which) {
    const bool fits = which ? plan_prefix(d, rows.data(), (int)rows.size(), groups.data(),
                                          (int)groups.size(), p)
                            : plan_pages(d, rows.data(), (int)rows.size(), n_pages, p);
    if (!fits) {
      CHECK(p.partial_rows > INT32_MAX);
      continue;
    }
    CHECK(p.ws_bytes >= 256 && p.off_lse + (size_t)p.partial_rows * 4 <= p.ws_bytes);
    CHECK(p.off_lse == (size_t)p.partial_rows * d.head_dim * 4);
    CHECK(p.piece >= 1 && (which || p.piece <= kListPages));
    std::vector<Range> parts;
    for (size_t i = 0; i < p.prefix.size(); ++i) {
      const PrefixRow& g = p.prefix[i];
      const int64_t turn = p.prefix[i].wide != kNarrow ? kWideTurn : kTurn;
      CHECK(g.n >= 1 && g.keys >= B && g.keys % B == 0 && g.split_keys >= 1);
      CHECK(g.n_split >= 1 && g.n_split <= kMaxGroupSplits);
      CHECK((int64_t)g.n_split * g.split_keys >= g.keys && (int64_t)(g.n_split - 1) * g.split_keys < g.keys);
      CHECK(g.n_split == 1 || g.split_keys % turn == 0);
      CHECK(g.part0 >= 0);
      parts.push_back({g.part0, (int64_t)g.n_split * g.n * hq});
      CHECK(prefix_items(g, hq / hkv, hkv) <= kMaxItems);
    }
    size_t at = 0;
    int32_t tok = 0, group = -1;
    int64_t own_parts = 0;
    bool split = false;
    for (const cp_row_meta& m : rows) {
      for (int32_t j = 0; j < m.chunk_len;) {
        CHECK(at < p.rows.size());
        const TokenRow& r = p.rows[at++];
        CHECK(r.tok0 == tok + j && r.start == m.chunk_start + j && r.req == m.req_id);
        CHECK(r.n >= 1 && r.n <= kPieceTokens && j + r.n <= m.chunk_len && r.n_split >= 1);
        CHECK(r.group >= -1 && r.group < (int64_t)p.prefix.size());
        int64_t own = std::min<int64_t>(n_pages, (r.start + r.n - 1) / B + 1);
        if (which) {
          own = (int64_t)r.start + r.n;
          if (r.group >= 0) {
            CHECK(r.group == group || (r.group == group + 1 && r.tok0 == p.prefix[r.group].tok0));
            group = r.group;
            const PrefixRow& g = p.prefix[r.group];
            CHECK(g.keys <= r.start && r.tok0 >= g.tok0 && r.tok0 + r.n <= g.tok0 + g.n);
            own -= g.keys;
          }
        } else {
          CHECK(r.group == -1);
        }
        CHECK(own >= 1 && r.n_split == (own - 1) / p.piece + 1);  // as the kernels have it
        const int64_t items = (int64_t)r.n_split * p.items_of(r.n) * hkv;
        CHECK(items <= kMaxItems && (int64_t)p.items_of(r.n) << p.log2_tokens >= r.n);
        CHECK(r.n_split == 1 || !which || p.piece % B == 0);
        own_parts += items * (hq / hkv) << p.log2_tokens;
        split |= r.n_split > 1 || r.group >= 0;
        j += r.n;
      }
      tok += m.chunk_len;
    }
    CHECK(at == p.rows.size() && split == p.parts);
    CHECK(p.unit_waves == 1 || p.unit_waves == 2 || p.unit_waves == 4 ||
          (p.unit_waves == kAllWaves && p.prefix.empty() && !p.parts));
    CHECK(p.log2_tokens == 0 || (which && hq / hkv << p.log2_tokens <= 16));
    if (split) parts.push_back({p.row_part0, own_parts});
    no_overlap(parts, p.partial_rows);
  }
}

}  // namespace

int main() {
  const int heads[][2] = {{1, 1}, {4, 2}, {8, 1}, {32, 8}, {64, 8}, {1024, 1024}, {8192, 1024}};
  for (int round = 0; round < 4000; ++round) {
    cp_attn_desc d{};
    const auto& h = heads[uniform(0, 6)];
    d.num_q_heads = h[0], d.num_kv_heads = h[1];
    d.head_dim = uniform(0, 1) ? 128 : 64, d.block_size = uniform(0, 1) ? 32 : 16;
    d.sm_scale = 0.1f;
    std::vector<cp_row_meta> rows;
    std::vector<cp_prefix_group> groups;
    const int n = spread(0, 300);
    const int32_t longest = spread(10, CP_CACHE_MAX_KEYS - 4096);
    const int32_t tokens = std::max<int64_t>(1, std::min<int64_t>(spread(1, 20000), kMaxPairs / h[0] / std::max(1, n)));
    while ((int)rows.size() < n) {
      const int32_t common = spread(0, longest);
      const int members = std::min<int>(n - (int)rows.size(), spread(1, 40));
      if (uniform(0, 3)) groups.push_back({(int32_t)rows.size(), members, common});
      for (int i = 0; i < members; ++i) {
        const int32_t start = (int32_t)std::min<int64_t>((int64_t)common + spread(0, longest), CP_CACHE_MAX_KEYS - 20000);
        const int32_t use = std::max(start, common);
        const int32_t len = (int32_t)std::min<int64_t>(uniform(0, 4) ? uniform(0, std::min(3, tokens)) : spread(0, tokens), CP_CACHE_MAX_KEYS - use);
        rows.push_back({(int32_t)rows.size(), use, len, use + len});
      }
    }
    check(d, rows, groups, spread(1, CP_CACHE_MAX_PAGES));
  }
  // the ends of the ranges
  for (int hkv : {1, 8, 1024})
    for (int g : {1, 8}) {
      cp_attn_desc d{};
      d.num_q_heads = hkv * g, d.num_kv_heads = hkv, d.head_dim = 128, d.block_size = 16;
      d.sm_scale = 0.1f;
      const int32_t K = CP_CACHE_MAX_KEYS, T = (int32_t)std::min<int64_t>(kMaxTokens, kMaxPairs / d.num_q_heads);
      check(d, {{0, K - 1, 1, K}}, {{0, 1, K - 1}}, 4096);
      check(d, {{0, K - 1, 1, K}}, {}, 1);
      check(d, {{0, K - T, T, K}}, {{0, 1, K - T}}, 4096);
      check(d, {{0, 0, T, T}}, {{0, 1, 0}}, 4096);
      std::vector<cp_row_meta> many;
      for (int32_t i = 0; i < 1000; ++i) many.push_back({i, K - 2, 1, K - 1});
      check(d, many, {{0, 1000, K - 2}}, 4096);
    }
  puts("ok");
  return 0;
}
