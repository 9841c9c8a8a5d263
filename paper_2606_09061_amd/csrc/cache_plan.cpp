// Plans of cp_page_select, cp_page_attn and cp_prefix_attn: the pieces of the rows
// and key ranges, and the workspace.
#include "cache_plan.hpp"

#include <algorithm>

#include "pieces.hpp"

namespace cpcache {

namespace {

using cptree::ceil_div;

// Work beyond so many workgroups is not cut: they fill the GPU eight times.
constexpr int64_t kUncut = 8 * cptree::kSlots;

// Waves of an item, of which the longest takes `turns`: four where the items alone
// do not fill the CUs' slots; one, which starts and ends once for all its keys,
// where they do, unless long items would end far apart.  us, 1 / 2 / 4 waves, lists
// of 64 pages on 32/8 heads: 256 items 48 / 31 / 29, 384 48 / 41 / 44, 512 52 / 54 /
// 56, 768 65 / 85 / 81, 1,024 95 / 104 / 106, 2,048 198 / 223 / 219; of 256 pages: 384
// 173 / 123 / 130, 512 186 / 165 / 165, 768 262 / 257 / 261, 2,048 739 / 681 / 667; 352
// items of 3 turns 25.7 / 19.4 / 20.6.
int unit_waves(int64_t items, int64_t turns) {
  if (items <= 320) return 4;
  if (items <= 512) return 2;
  return items <= 1536 || turns <= 16 ? 1 : 4;
}

// Whether items of so many turns, uncut, are done in one launch, by eight waves each:
// where cutting and merging them takes as long.  us in a graph, so / cut or with fewer
// waves, lists on 32/8 heads of 64: 32 pages (4 turns), 8 items 6.0 / 6.3, 64 items 6.8 /
// 7.7; 64 pages, 8 items 7.3 / 8.3, 64 items 9.7 / 11.8, 256 items 15.6 / 17.4; 128 pages,
// 8 items 11.4 / 8.6, 64 items 15.1 / 13, 128 items 18.8 / 20.6; 256 pages, 128 items 31.6 /
// 33.  Heads of 128: 64 pages, 8 items 9.4 / 9.0 (a launch less is worth 1.6 to the
// host), 16 items 11.4 / 10.0, 64 items 16.6 / 14.0.
bool whole(int d, int64_t items, int64_t turns) {
  if (d == 64) return items <= 256 && (turns <= 8 || (items >= 128 && turns <= 32));
  return items <= 8 && turns <= 8;
}
// Whether tokens of groups read all of their keys so, common ones too, which the
// caches hold then.  us, so / the groups' keys once, 32/8 heads of 128, 4 requests: 128
// keys in common 5.3 / 8.6, 500 8.0 / 10.1, 1,000 10.7 / 10.3 (eager 10.2 / 11.0), 2,000 17.7 /
// 10.7; 32 requests: 500 8.5 / 12.8, 1,000 10.8 / 14.2, 2,000 17.9 / 17.4; 64 requests: 128
// 10.4 / 12.8, 500 16.6 / 17.3.  4/2 heads of 64, 4 requests: 500 5.9 / 8.0, 1,000 8.3 /
// 8.2 (8.4 / 11.1); 64 requests: 500 7.4 / 8.9.
bool ungrouped(int64_t items, int64_t turns) { return items <= 256 && turns <= 8; }

// Times of the attention kernels (pieces.hpp), in us; `merged`: with a merge in any case.
cptree::Cost cost_of(int d, bool wide, bool merged, double memory) {
  const double x = d / 128.0, merge = merged ? 0.0 : 4.5;
  if (wide) return {kWideTurn, 0.4 + 2.2 * x, 1.0 + 0.2 * x, 7.0, merge, 0.2 * x, memory};
  return {kTurn, 5.5 * x, 0.3 + 1.2 * x, 3.2, merge, 0.3 * x, memory};
}

// A narrow workgroup starts and ends sooner, a wide one takes four times the rows
// and reads K and V for all of them: groups of up to kWideTile rows stay narrow while
// there are few common keys in all.  us, narrow / wide, on 32/8 heads: one group of 36
// rows and 256 keys 11.0 / 12.5, 1,000 keys 11.7 / 13.6, 4,000 keys 16.3 / 15.8, 16,000
// keys 31 / 26; of 128 rows 13.5 / 14.8, 15.7 / 17.1, 23.6 / 19.6, 53 / 31; 8 groups of
// 36 rows and 256 keys 19.9 / 15.9.
constexpr double kNarrowKeys = 1536;
// Common K and V beyond which groups of one wide tile read them past the caches: 8
// groups of 128 rows and 4,096 keys on 64/8 heads, 134 MB, 49 -> 43 us; one of 8,192
// on 32/8, 34 MB, 25.1 -> 25.8.
constexpr double kStreamBytes = 64e6;

// us that keys take to come from memory
double memory_us(const cp_attn_desc& d, double keys) {
  return keys * d.num_kv_heads * d.head_dim * 4.0 / 5.3e6;
}

// Turns of a piece: the tree plan's choice or a somewhat longer piece, whose fewer
// partial rows may be worth more than CUs that stay idle.
int piece_of(const cptree::Work& w, const cptree::Cost& c) {
  double time = 0;
  const int chosen = cptree::best_piece(w, c, &time);
  int best = chosen;
  for (const int piece : {chosen * 5 / 4, chosen * 3 / 2, chosen * 2}) {
    const double t = cptree::time_of(cptree::load_of(w, piece), c);
    if (t < time) time = t, best = piece;
  }
  return std::max(1, best);
}

// Adds a row, in pieces of kPieceTokens tokens.
void add_row(AttnPlan& out, int32_t tok0, const cp_row_meta& m, int32_t group) {
  for (int32_t j = 0; j < m.chunk_len; j += kPieceTokens)
    out.rows.push_back(TokenRow{tok0 + j, std::min(kPieceTokens, m.chunk_len - j),
                                m.chunk_start + j, m.req_id, group, 1});
}

void reset(AttnPlan& out) {
  out.rows.clear(), out.prefix.clear();
  out.log2_tokens = 0, out.piece = 1, out.parts = false, out.row_part0 = 0;
  out.partial_rows = 0, out.off_lse = 0, out.ws_bytes = 256;
}

// Cuts the rows' ranges, own(row) units of which `per_turn` make a turn and
// `most` may make a piece (`one`: in no case), and lays out the workspace.
template <class Own>
bool cut_rows(AttnPlan& out, const cp_attn_desc& d, double keys, int per_turn, int most, bool one,
              Own&& own) {
  thread_local cptree::Work work;
  work.turns.clear(), work.per_split.clear(), work.partial.clear();
  int64_t uncut = 0, all = 0;
  for (const TokenRow& r : out.rows)
    uncut += (int64_t)out.items_of(r.n) * d.num_kv_heads, all = std::max<int64_t>(all, own(r));
  out.piece = most;
  if (one || (out.prefix.empty() && whole(d.head_dim, uncut, ceil_div(all, per_turn)))) {
    out.unit_waves = kAllWaves;
    return true;
  }
  if (uncut < kUncut && !out.rows.empty()) {
    for (const TokenRow& r : out.rows) {
      work.turns.push_back((uint32_t)ceil_div(own(r), per_turn));
      work.per_split.push_back(out.items_of(r.n) * d.num_kv_heads);
      work.partial.push_back(r.n * d.num_q_heads);
    }
    const int turns = piece_of(work, cost_of(d.head_dim, false, !out.prefix.empty(), memory_us(d, keys)));
    out.piece = (int)std::min<int64_t>(most, (int64_t)turns * per_turn);
  }
  int64_t partial = 0, items = 0, longest = 0;
  for (TokenRow& r : out.rows) {
    r.n_split = (int)ceil_div(own(r), out.piece);
    out.parts |= r.n_split > 1 || r.group >= 0;
    const int64_t mine = (int64_t)r.n_split * out.items_of(r.n) * d.num_kv_heads;
    partial += (mine * (d.num_q_heads / d.num_kv_heads)) << out.log2_tokens;
    items += mine;
    longest = std::max<int64_t>(longest, ceil_div(std::min<int64_t>(own(r), out.piece), per_turn));
  }
  out.unit_waves = unit_waves(items, longest);
  out.row_part0 = (int32_t)std::min<int64_t>(out.partial_rows, INT32_MAX);
  if (out.parts) out.partial_rows += partial;
  if (out.partial_rows > INT32_MAX) return false;
  out.off_lse = (size_t)out.partial_rows * d.head_dim * 4;
  out.ws_bytes = std::max<size_t>(256, out.off_lse + (size_t)out.partial_rows * 4);
  return true;
}

// Cuts the common keys of the groups that one of the kernels takes.
void cut_groups(AttnPlan& out, const cp_attn_desc& d, bool wide) {
  const int G = d.num_q_heads / d.num_kv_heads, turn = wide ? kWideTurn : kTurn;
  thread_local cptree::Work work;
  work.turns.clear(), work.per_split.clear(), work.partial.clear();
  int64_t uncut = 0;
  double keys = 0;
  for (size_t i = 0; i < out.prefix.size(); ++i)
    if ((out.prefix[i].wide != kNarrow) == wide) {
      uncut += prefix_items(out.prefix[i], G, d.num_kv_heads);
      keys += out.prefix[i].keys;
    }
  if (uncut == 0) return;
  int piece = INT32_MAX / turn;
  if (uncut < kUncut) {
    for (size_t i = 0; i < out.prefix.size(); ++i) {
      const PrefixRow& p = out.prefix[i];
      if ((out.prefix[i].wide != kNarrow) != wide) continue;
      work.turns.push_back((uint32_t)ceil_div(p.keys, turn));
      work.per_split.push_back((uint32_t)prefix_items(p, G, d.num_kv_heads));
      work.partial.push_back((uint32_t)((int64_t)p.n * d.num_q_heads));
    }
    piece = piece_of(work, cost_of(d.head_dim, wide, true, memory_us(d, keys)));
  }
  for (size_t i = 0; i < out.prefix.size(); ++i) {
    PrefixRow& p = out.prefix[i];
    if ((out.prefix[i].wide != kNarrow) != wide) continue;
    const int64_t turns = ceil_div(p.keys, turn);
    const int64_t per = ceil_div(turns, std::min<int64_t>(kMaxGroupSplits, ceil_div(turns, piece)));
    p.n_split = (int32_t)ceil_div(turns, per);
    p.split_keys = (int32_t)std::min<int64_t>(per * turn, INT32_MAX);
  }
}

// Pages that a workgroup scores: a turn of its waves (64 pages of head_dim 128), and
// as many more as leave kScoreItems workgroups.
constexpr int kLeastChunk = 64, kMostChunk = 512;
constexpr int64_t kScoreItems = 1024;
// How one launch does both, a workgroup each (token, kv head), if it does: of four waves
// for few pages or many (token, kv head)s, of 8 or 16 where there are about as many of
// these as CUs.  us, 32/8 heads of 128, in two launches / by 4 waves / by 16, n (token, kv
// head)s: n 8, 63 pages 8.4 / 5.9 / 6.9, 125 8.5 / 7.2 / 8.7, 188 8.8 / 8.6 / 9.1, 250 8.8 /
// 10.0 / 10.4; n 128, 125 9.7 / 8.2 / 9.6, 250 12.1 / 12.0 / 11.9, 475 15.7 / 19.5 / 17.1;
// n 256, 250 15.8 / 13.4 / 13.1, 475 24.5 / 21.7 / 18.9, 1,000 38.1 / 38.2 / 31.1; n 384, 250
// 21.2 / 18.3 / 23.3, 1,000 47.5 / 52.0 / 56.0; n 512, 475 37.5 / 29.9 / 37.2; n 2,048, 125
// 61.8 / 48.3 / 85.8.  Of uneven numbers of pages the largest sets the time: up to 500, n
// 256 20.1 / 20.6 / 17.9, n 512 30.2 / 29.6 / 34.0; up to 1,000, n 512 47.9 / 51.0 / 54.3.
// (By 16 waves up to 4,096: 256 x 2,000 60.6 / 56.9, uneven 62 / 73.)  64/8 heads, n 8:
// 125 9.3 / 8.8, 188 9.6 / 10.8.  16/16 heads of 64: n 16, 250 8.3 / 6.7; n 1,024, up to
// 1,000 50.3 / 44.0.
One in_one(const cp_attn_desc& d, int64_t n, int most) {
  const bool half = d.head_dim == 64, heavy = d.num_q_heads >= 8 * d.num_kv_heads;
  if (most <= 256)
    return n >= 112 || half || most <= (heavy ? 128 : 176) ? One::kFour256 : One::kNo;
  if (n > 256) return most <= (half ? 1024 : 512) ? One::kFour1024 : One::kNo;
  return n > 128 && most <= 1024 ? One::kAll1024 : One::kNo;
}

}  // namespace

void plan_select(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, int32_t n_pages,
                 SelectPlan& out) {
  const int hkv = desc.num_kv_heads;
  out.rows.clear(), out.scores = 0, out.most = 0;
  int32_t tok = 0;
  for (int32_t r = 0; r < n_rows; ++r) {
    const cp_row_meta& m = rows[r];
    if (m.chunk_len == 0) continue;
    const int32_t held = (m.ctx_len - 1) / desc.block_size + 1;
    const int32_t stride = held > n_pages ? held : 0;  // 0: no token has to choose
    out.most = std::max(out.most, held);
    // a piece's workgroups of the scores fit a launch
    const int64_t chunks = std::max(1, (stride + kLeastChunk - 1) / kLeastChunk);
    const int32_t step = (int32_t)std::max<int64_t>(
        1, std::min<int64_t>(kPieceTokens, kMaxItems / 2 / (chunks * hkv)));
    for (int32_t j = 0; j < m.chunk_len; j += step) {
      const int32_t n = std::min(step, m.chunk_len - j);
      out.rows.push_back(
          SelectRow{0, tok + j, n, m.chunk_start + j, m.req_id, stride, out.scores});
      out.scores += (int64_t)n * hkv * stride;
    }
    tok += m.chunk_len;
  }
  out.chunk = kLeastChunk;
  // (a token's scores fit a launch, whatever its pages and heads)
  while ((out.chunk < kMostChunk && out.scores > 2 * out.chunk * kScoreItems) ||
         (int64_t)hkv * (out.most / out.chunk + 1) > kMaxItems / 2)
    out.chunk *= 2;
  out.one = in_one(desc, (int64_t)tok * hkv, out.most);
}

bool plan_pages(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, int32_t n_pages,
                AttnPlan& out) {
  reset(out);
  const int64_t B = desc.block_size;
  const auto listed = [&](const TokenRow& r) {  // of the piece's last token
    return std::min<int64_t>(n_pages, (r.start + r.n - 1) / B + 1);
  };
  int32_t tok = 0;
  double keys = 0;
  for (int32_t i = 0; i < n_rows; ++i) {
    add_row(out, tok, rows[i], -1);
    tok += rows[i].chunk_len;
  }
  for (const TokenRow& r : out.rows) keys += (double)r.n * listed(r) * B;
  return cut_rows(out, desc, keys, kTurn / desc.block_size, kListPages, false, listed);
}

bool plan_prefix(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows,
                 const cp_prefix_group* groups, int32_t n_groups, AttnPlan& out) {
  reset(out);
  const int hq = desc.num_q_heads, G = hq / desc.num_kv_heads, B = desc.block_size;
  int64_t items = 0, most = 0;
  for (int32_t i = 0; i < n_rows; ++i)
    if (rows[i].chunk_len > 0) {
      items += (int64_t)rows[i].chunk_len * desc.num_kv_heads;
      most = std::max<int64_t>(most, rows[i].ctx_len);
    }
  const bool one = n_groups > 0 && ungrouped(items, ceil_div(most, kTurn));
  if (one) n_groups = 0;
  int32_t tok = 0, g = 0, last = -1;
  for (int32_t i = 0; i < n_rows; ++i) {
    while (g < n_groups && i >= groups[g].first_row + groups[g].n_rows) ++g;
    int32_t ref = -1;
    if (g < n_groups && i >= groups[g].first_row && groups[g].common >= B && rows[i].chunk_len > 0) {
      if (last != g) {
        const int32_t keys = groups[g].common / B * B;
        out.prefix.push_back(PrefixRow{0, tok, 0, rows[i].req_id, keys, 1, keys, 0, 0, 0, 0});
        last = g;
      }
      ref = (int32_t)out.prefix.size() - 1;
      out.prefix.back().n += rows[i].chunk_len;
    }
    add_row(out, tok, rows[i], ref);
    tok += rows[i].chunk_len;
  }
  double common = 0;
  for (const PrefixRow& p : out.prefix) common += p.keys;
  const bool large = common * desc.num_kv_heads * desc.head_dim * 4.0 > kStreamBytes;
  const int64_t narrow = common <= kNarrowKeys ? kWideTile : kNarrowTile;
  for (PrefixRow& p : out.prefix) {
    const int64_t m = (int64_t)p.n * G;
    p.wide = m <= narrow ? kNarrow : m <= kWideTile && large ? kStreamed : kCached;
  }
  cut_groups(out, desc, false);
  cut_groups(out, desc, true);
  for (PrefixRow& p : out.prefix) {
    p.part0 = (int32_t)std::min<int64_t>(out.partial_rows, INT32_MAX);
    out.partial_rows += (int64_t)p.n_split * p.n * hq;
  }
  for (const TokenRow& r : out.rows)  // 16 columns at most
    while (r.n > (1 << out.log2_tokens) && ((2 * G) << out.log2_tokens) <= 16) ++out.log2_tokens;
  const auto own = [&](const TokenRow& r) {
    return (int64_t)r.start + r.n - (r.group < 0 ? 0 : out.prefix[r.group].keys);
  };
  double keys = 0;
  for (const TokenRow& r : out.rows) keys += (double)own(r);
  return cut_rows(out, desc, keys, kTurn, INT32_MAX / kTurn * kTurn, one, own);
}

}  // namespace cpcache
