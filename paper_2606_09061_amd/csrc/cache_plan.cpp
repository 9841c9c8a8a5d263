// Plans of cp_page_attn and cp_prefix_attn: the pieces of the key ranges and the
// workspace.
#include "cache_plan.hpp"

#include <algorithm>

#include "pieces.hpp"

namespace cpcache {

namespace {

using cptree::ceil_div;

// Work beyond so many workgroups is not cut: they fill the GPU eight times.
constexpr int64_t kUncut = 8 * cptree::kSlots;

// Times as measured of the attention kernel (pieces.hpp), in us.
cptree::Cost cost_of(int d, double memory) {
  const double x = d / 128.0;
  return {kTurn, 5.5 * x, 0.3 + 1.2 * x, 3.2, 5.5, 0.3 * x, memory};
}

// Turns of a piece, for rows of (turns, workgroups per piece, partial rows per piece).
int piece_of(const cptree::Work& w, int d, double memory) {
  double time = 0;
  return std::max(1, cptree::best_piece(w, cost_of(d, memory), &time));
}

// Adds a row, in pieces of kPieceTokens tokens.
void add_row(AttnPlan& out, int32_t tok0, const cp_row_meta& m, int32_t group) {
  for (int32_t j = 0; j < m.chunk_len; j += kPieceTokens)
    out.rows.push_back(AttnRow{0, tok0 + j, std::min(kPieceTokens, m.chunk_len - j),
                               m.chunk_start + j, m.req_id, group, 1, 0});
}

void reset(AttnPlan& out) {
  out.rows.clear(), out.prefix.clear(), out.groups.clear();
  out.piece = 1, out.partial_rows = 0, out.off_lse = 0, out.ws_bytes = 256;
}

bool finish(AttnPlan& out, int d) {
  if (out.partial_rows > INT32_MAX) return false;
  out.off_lse = (size_t)out.partial_rows * d * 4;
  out.ws_bytes = std::max<size_t>(256, out.off_lse + (size_t)out.partial_rows * 4);
  return true;
}

// n_split and the partial rows of rows whose piece is known; own(row) is the
// length of its range in units of the piece.
template <class Own>
void cut_rows(AttnPlan& out, int hq, Own&& own) {
  for (AttnRow& r : out.rows) {
    r.n_split = (int)std::max<int64_t>(1, ceil_div(own(r), out.piece));
    if (r.n_split == 1) continue;
    r.part0 = (int32_t)std::min<int64_t>(out.partial_rows, INT32_MAX);
    out.partial_rows += (int64_t)r.n_split * r.n * hq;
  }
}

}  // namespace

bool plan_pages(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, int32_t n_pages,
                AttnPlan& out) {
  reset(out);
  const int64_t B = desc.block_size;
  const int per_turn = kTurn / desc.block_size;
  thread_local cptree::Work work;
  work.turns.clear(), work.per_split.clear(), work.partial.clear();
  int32_t tok = 0;
  int64_t uncut = 0;
  double pages = 0;
  const auto listed = [&](const AttnRow& r) {  // of the piece's last token
    return std::min<int64_t>(n_pages, (r.start + r.n - 1) / B + 1);
  };
  for (int32_t i = 0; i < n_rows; ++i) {
    add_row(out, tok, rows[i], -1);
    tok += rows[i].chunk_len;
  }
  for (const AttnRow& r : out.rows) {
    uncut += (int64_t)r.n * desc.num_kv_heads;
    pages += (double)r.n * listed(r);
  }
  out.piece = kListPages;
  if (uncut < kUncut) {
    for (const AttnRow& r : out.rows) {
      work.turns.push_back((uint32_t)ceil_div(listed(r), per_turn));
      work.per_split.push_back(r.n * desc.num_kv_heads);
      work.partial.push_back(r.n * desc.num_q_heads);
    }
    if (!out.rows.empty())
      out.piece = std::min(kListPages,
                           per_turn * piece_of(work, desc.head_dim,
                                               pages * B * desc.num_kv_heads * desc.head_dim * 4.0 /
                                                   5.3e6));
  }
  cut_rows(out, desc.num_q_heads, listed);
  return finish(out, desc.head_dim);
}

bool plan_prefix(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows,
                 const cp_prefix_group* groups, int32_t n_groups, AttnPlan& out) {
  reset(out);
  const int hq = desc.num_q_heads, hkv = desc.num_kv_heads, G = hq / hkv, B = desc.block_size;
  const double per_key = hkv * desc.head_dim * 4.0 / 5.3e6;
  thread_local cptree::Work work;
  // the groups' common keys
  int32_t tok = 0, g = 0;
  for (int32_t i = 0; i < n_rows; ++i) {
    while (g < n_groups && i >= groups[g].first_row + groups[g].n_rows) ++g;
    int32_t ref = -1;
    if (g < n_groups && i >= groups[g].first_row && groups[g].common >= B && rows[i].chunk_len > 0) {
      if (out.prefix.empty() || out.prefix.back().item0 != g) {  // (the group, for now)
        const int32_t keys = groups[g].common / B * B;
        out.prefix.push_back(PrefixRow{g, tok, 0, rows[i].req_id, keys, 1, keys, 0});
        out.groups.push_back(GroupRef{keys, 0, 1, 0, tok, 0});
      }
      ref = (int32_t)out.groups.size() - 1;
      out.prefix.back().n += rows[i].chunk_len;
    }
    add_row(out, tok, rows[i], ref);
    tok += rows[i].chunk_len;
  }
  int64_t uncut = 0;
  double keys = 0;
  const auto tiles = [&](const PrefixRow& p) { return ceil_div((int64_t)p.n * G, kPrefixTile); };
  for (const PrefixRow& p : out.prefix) uncut += tiles(p) * hkv, keys += (double)p.keys;
  int piece = INT32_MAX / kTurn;
  work.turns.clear(), work.per_split.clear(), work.partial.clear();
  if (uncut < kUncut && !out.prefix.empty()) {
    for (const PrefixRow& p : out.prefix) {
      work.turns.push_back((uint32_t)ceil_div(p.keys, kTurn));
      work.per_split.push_back((uint32_t)(tiles(p) * hkv));
      work.partial.push_back((uint32_t)std::min<int64_t>((int64_t)p.n * hq, UINT32_MAX));
    }
    piece = piece_of(work, desc.head_dim, keys * per_key);
  }
  for (size_t i = 0; i < out.prefix.size(); ++i) {
    PrefixRow& p = out.prefix[i];
    const int64_t turns = ceil_div(p.keys, kTurn);
    int64_t n = std::min<int64_t>(kMaxGroupSplits, ceil_div(turns, piece));
    const int64_t per = ceil_div(turns, n);
    n = ceil_div(turns, per);
    p.n_split = (int32_t)n;
    p.split_keys = (int32_t)std::min<int64_t>(per * kTurn, INT32_MAX);
    p.part0 = (int32_t)std::min<int64_t>(out.partial_rows, INT32_MAX);
    out.partial_rows += n * p.n * hq;
    out.groups[i] = GroupRef{p.keys, p.part0, p.n_split, p.n * G, p.tok0, 0};
  }
  // every token's own keys
  const auto own = [&](const AttnRow& r) {
    return (int64_t)r.start + r.n - (r.group < 0 ? 0 : out.groups[r.group].keys);
  };
  uncut = 0, keys = 0;
  for (const AttnRow& r : out.rows) uncut += (int64_t)r.n * hkv, keys += (double)own(r);
  out.piece = INT32_MAX;
  work.turns.clear(), work.per_split.clear(), work.partial.clear();
  if (uncut < kUncut && !out.rows.empty()) {
    for (const AttnRow& r : out.rows) {
      work.turns.push_back((uint32_t)ceil_div(own(r), kTurn));
      work.per_split.push_back(r.n * hkv);
      work.partial.push_back(r.n * hq);
    }
    out.piece = (int)std::min<int64_t>(INT32_MAX, (int64_t)kTurn *
                                       piece_of(work, desc.head_dim, keys * per_key));
  }
  cut_rows(out, hq, own);
  return finish(out, desc.head_dim);
}

}  // namespace cpcache
