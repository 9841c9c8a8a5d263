// Random batches through the launches of libcpcache's selection and attention: every
// workgroup is launched once, and every grid has fewer than 2^32 threads.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "cache_batches.hpp"

using namespace cpcache;

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      fprintf(stderr, "line %d: %s\n", __LINE__, #x);         \
      exit(1);                                                \
    }                                                         \
  } while (0)

namespace {

std::mt19937_64 rng(11);

int64_t uniform(int64_t lo, int64_t hi) {
  return std::uniform_int_distribution<int64_t>(lo, hi)(rng);
}

int32_t spread(int64_t lo, int64_t hi) {  // over the logarithm
  const double a = std::uniform_real_distribution<double>(std::log(lo + 1.0), std::log(hi + 1.0))(rng);
  return (int32_t)std::min<int64_t>(hi, std::max<int64_t>(lo, (int64_t)(std::exp(a) - 1.0)));
}

void grid(int64_t workgroups, int64_t threads) {
  CHECK(workgroups >= 1 && workgroups < (1ll << 31) && workgroups * threads < (1ll << 32));
}

// Launches of pieces whose tokens follow one another; returns the workgroups.
struct Pieces {
  int64_t tok = -1, items = 0;
  void add(const SelectRows& b, int n, int64_t launched, int64_t threads) {
    grid(launched, threads);
    CHECK(n >= 1 && n <= kSelectRows);
    for (int i = 0; i < kSelectRows; ++i) {
      const SelectRow& r = b.r[i];
      if (i >= n) {
        CHECK(r.item0 == INT_MAX);
        continue;
      }
      CHECK(r.tok0 > tok && r.n >= 1 && (i == 0 ? r.item0 == 0 : r.item0 > b.r[i - 1].item0));
      CHECK(r.item0 < launched);
      tok = r.tok0 + r.n - 1;
    }
    items += launched;
  }
};

void check_select(const cp_attn_desc& d, const std::vector<cp_row_meta>& rows, int32_t n_pages) {
  static SelectPlan p;
  plan_select(d, rows.data(), (int)rows.size(), n_pages, p);
  const int64_t hkv = d.num_kv_heads;
  int64_t tokens = 0, scored = 0;
  for (const SelectRow& r : p.rows) {
    tokens += r.n;
    if (r.stride > 0) scored += r.n * hkv * ((r.stride + p.chunk - 1) / p.chunk);
  }
  // the threads of select_kernel and choose_kernel
  const int64_t threads = p.one == One::kAll1024 ? 1024
                          : p.one != One::kNo    ? 256
                          : p.most > 1024 && p.most <= 16384 ? 1024 : 256;
  Pieces score, choice;
  bool begun = false;
  CHECK(select_launches(
            d, p,
            [&](SelectRows& b, int n, int items) {
              CHECK(!begun && p.one == One::kNo);
              score.add(b, n, items, 256);
              return CP_OK;
            },
            [&](SelectRows& b, int n, int items) {
              begun = true;
              choice.add(b, n, items, threads);
              return CP_OK;
            }) == CP_OK);
  CHECK(choice.items == tokens * hkv && score.items == (p.one == One::kNo ? scored : 0));
}

void check_attn(const cp_attn_desc& d, const AttnPlan& p) {
  const int64_t hkv = d.num_kv_heads, G = d.num_q_heads / hkv;
  size_t r = 0;
  int64_t groups = 0, part = p.row_part0;
  CHECK(attn_launches(d, p, [&](const AttnLaunch& x) {
          CHECK(x.n >= 1 && x.n <= kAttnRows && x.n_groups <= kGroups);
          const int64_t per = std::max(1, 4 / p.unit_waves);
          grid(x.group_items + (x.items + per - 1) / per, 64 * std::max(4, p.unit_waves));
          const int share = merge_share(d, x.n_tokens, x.most);
          if (x.merge) grid(merge_items(d, x.n_tokens, share), 256);
          CHECK(x.part0 == part);
          int64_t items = 0, tok = p.rows[r].tok0;
          for (int i = 0; i < x.n; ++i, ++r) {
            const TokenRow& t = p.rows[r];
            CHECK(x.b.r[i].tok0 == t.tok0 && t.tok0 == tok && x.b.r[i].start == t.start);
            CHECK(x.b.r[i].item0 == items);
            items += (int64_t)t.n_split * p.items_of(t.n) * hkv;
            tok += t.n;
            int in = -1;
            for (int g = 0; g < x.n_groups; ++g)
              if (x.b.g[g].row0 <= i && i < x.b.g[g].row1) in = in < 0 ? g : INT_MAX;
            CHECK(in == -1 ? t.group < 0 : in != INT_MAX && t.group >= 0);
            if (in >= 0) CHECK(x.b.g[in].part0 == p.prefix[t.group].part0);
            CHECK(t.n_split == 1 && t.group < 0 ? true : x.merge);
          }
          CHECK(items == x.items && x.b.r[x.n].tok0 == tok && x.b.r[x.n].item0 == INT_MAX);
          CHECK(tok - p.rows[r - x.n].tok0 == x.n_tokens);
          int64_t shared = 0;  // groups whose first row is here
          for (int g = 0; g < x.n_groups; ++g) {
            const TokenRow& t = p.rows[r - x.n + x.b.g[g].row0];
            CHECK(x.b.g[g].item0 == shared);
            if (t.tok0 == p.prefix[t.group].tok0)
              shared += prefix_items(p.prefix[t.group], (int)G, (int)hkv), ++groups;
          }
          CHECK(shared == x.group_items);
          if (p.parts) part += (items * G) << p.log2_tokens;
          return CP_OK;
        }) == CP_OK);
  CHECK(r == p.rows.size() && groups == (int64_t)p.prefix.size());
  CHECK(!p.parts || part == p.partial_rows);
}

void check(const cp_attn_desc& d, const std::vector<cp_row_meta>& rows,
           const std::vector<cp_prefix_group>& groups, int32_t n_pages) {
  static AttnPlan p;
  check_select(d, rows, n_pages);
  if (plan_pages(d, rows.data(), (int)rows.size(), n_pages, p)) check_attn(d, p);
  if (plan_prefix(d, rows.data(), (int)rows.size(), groups.data(), (int)groups.size(), p))
    check_attn(d, p);
}

// Groups of (rows, tokens in common) that take these kernels.
void check_kinds(const cp_attn_desc& d, const std::vector<std::vector<int32_t>>& sizes) {
  std::vector<cp_row_meta> rows;
  std::vector<cp_prefix_group> groups;
  for (const auto& g : sizes) {
    groups.push_back({(int32_t)rows.size(), g[0], g[1]});
    for (int32_t i = 0; i < g[0]; ++i) rows.push_back({(int32_t)rows.size(), g[1] + i, 1, g[1] + i + 1});
  }
  AttnPlan p;
  CHECK(plan_prefix(d, rows.data(), (int)rows.size(), groups.data(), (int)groups.size(), p));
  CHECK(p.prefix.size() == sizes.size());
  for (size_t i = 0; i < sizes.size(); ++i) CHECK(p.prefix[i].wide == sizes[i][2]);
}

cp_attn_desc desc(int hq, int hkv, int head_dim, int block) {
  cp_attn_desc d{};
  d.num_q_heads = hq, d.num_kv_heads = hkv, d.head_dim = head_dim, d.block_size = block;
  d.sm_scale = 0.1f;
  return d;
}

}  // namespace

int main() {
  const int heads[][2] = {{1, 1}, {4, 2}, {8, 1}, {32, 8}, {64, 8}, {128, 128}, {1024, 1024}, {8192, 1024}};
  for (int round = 0; round < 3000; ++round) {
    const auto& h = heads[uniform(0, 7)];
    const cp_attn_desc d = desc(h[0], h[1], uniform(0, 1) ? 128 : 64, uniform(0, 1) ? 32 : 16);
    std::vector<cp_row_meta> rows;
    std::vector<cp_prefix_group> groups;
    const int n = spread(1, 400);
    const int32_t longest = spread(10, CP_CACHE_MAX_KEYS / 4);
    const int32_t most = (int32_t)std::max<int64_t>(1, std::min<int64_t>({spread(1, 70000), kMaxPairs / h[0] / n, kMaxTokens / n}));
    while ((int)rows.size() < n) {
      const int32_t common = spread(0, longest);
      const int members = std::min<int>(n - (int)rows.size(), spread(1, 200));
      if (uniform(0, 3)) groups.push_back({(int32_t)rows.size(), members, common});
      for (int i = 0; i < members; ++i) {
        const int32_t start = common + spread(0, longest);
        const int32_t len = uniform(0, 3) ? (int32_t)uniform(0, std::min(3, most)) : (int32_t)uniform(0, most);
        rows.push_back({(int32_t)rows.size(), start, len, start + len});
      }
    }
    check(d, rows, groups, spread(1, CP_CACHE_MAX_PAGES));
  }
  // the ends of the ranges: launches of 1,024 threads for many (token, kv head)s, and
  // merges of 2^27 (token, q head)s
  for (int pages : {1000, 1025, 4096, 4097, 16384, 16385})
    for (int hkv : {73, 74, 128, 1024}) {
      const cp_attn_desc d = desc(hkv, hkv, 128, 16);
      const int32_t T = (int32_t)std::min<int64_t>(60000, kMaxPairs / hkv), ctx = std::max(T, 16 * pages);
      check(d, {{0, ctx - T, T, ctx}}, {}, 4);
      check(d, {{0, 16 * pages - 1, 1, 16 * pages}, {1, 0, T - 1, T - 1}}, {}, 4);
      std::vector<cp_row_meta> many;
      for (int32_t i = 0; i < 120 && 500 * 120 <= T; ++i) many.push_back({i, 16 * pages - 500, 500, 16 * pages});
      check(d, many, {}, 4);
    }
  for (int head_dim : {64, 128})
    for (int hkv : {1, 8, 1024})
      for (int g : {1, 8}) {
        const cp_attn_desc d = desc(hkv * g, hkv, head_dim, 16);
        const int32_t T = (int32_t)std::min<int64_t>(kMaxTokens, kMaxPairs / (hkv * g)), K = 1 << 24;
        check(d, {{0, K - T, T, K}}, {{0, 1, K - T}}, 4096);
        check(d, {{0, K - T, T, K}}, {}, 300);
        check(d, {{0, K - 1, 1, K}, {1, K - T, T - 1, K - 1}}, {{0, 2, K - T}}, 1);
      }
  // the groups of tests/test_gpu_cache_far.py
  check_kinds(desc(8, 1, 128, 16), {{5, 100000, kStreamed}, {17, 20003, kCached}, {3, 6001, kNarrow}});
  check_kinds(desc(32, 4, 64, 32), {{6, 50001, kStreamed}, {20, 10000, kCached}, {4, 4005, kNarrow}});
  check_kinds(desc(8, 8, 128, 32), {{40, 14000, kStreamed}, {130, 1700, kCached}, {3, 1800, kNarrow}});
  check_kinds(desc(4, 2, 128, 16), {{31, 60003, kStreamed}, {70, 3000, kCached}, {5, 2040, kNarrow}});
  check_kinds(desc(64, 8, 128, 16), {{6, 16000, kStreamed}, {20, 1700, kCached}, {2, 900, kNarrow}});
  puts("ok");
  return 0;
}
