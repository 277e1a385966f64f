// Host plan of the chunk attention (dbsa_chunk_attn): which rows walk which runs of keys, dealt to persistent
// workers.  Integer work only, no GPU calls.
//
// Every new token of a question attends the sink, the question's selected groups and its own keys.  A UNIT is a block
// of tokens (times the query heads of a KV head: the rows of a workgroup) with one list of KV tiles:
//   * a question whose chunk fills a workgroup's rows walks its lists by itself, block of tokens by block of tokens:
//     sink, selected groups, own keys, one softmax state from the first tile to the last;
//   * the tokens of all smaller chunks are gathered per segment (Sec. 2.2: the caches of the selected groups are used
//     in place by every question that selected them), so that a group's keys are fetched once for as many of its users
//     as the rows hold; their own keys are units of their own, and a merge pass joins the softmax states.
// The units, laid end to end, are dealt to W workers per KV head in equal shares: a unit that does not fit a worker's
// share is cut there, and what is cut is merged.
#include <algorithm>
#include <climits>

#include "layout.hpp"

namespace {

// workgroups of rows rows, per_cu to a compute unit, and what a tile costs one
struct ChunkShape {
  int32_t rows, per_cu, tile_cost;
};

struct Unit {
  int32_t tok_begin, n_tok;  // in ck_toks
  int32_t ent_begin, n_ent;  // pool tiles, in ck_ent
  int32_t own_u, own_tiles;  // question whose own keys follow them (-1: none), and their expected tiles
  int64_t cost() const { return int64_t{n_ent} + own_tiles; }
};

// What starting and finishing a record costs, in tiles: its rows of Q, the first tiles' latency, the partial states.  (128 questions
// of 4 tokens, 7 records to a worker: 376 us with 2, 372 with 3, 375 with 4, 391 with 6.)
constexpr int64_t kRecordCost = 3;
// Tiles of a unit that is not worth cutting: the merge's launch costs 6 us, a tile of a lone workgroup 2.
constexpr int64_t kShortUnit = 3;

}  // namespace

int dbsa_build_chunk_lists(const dbsa_pool_desc* pool, const dbsa_select_desc* sel, int32_t n_q_heads, int32_t n_kv_heads,
                           const int32_t* own_tokens, dbsa_layout* L) {
  if (!pool || !sel || !L || n_q_heads < 1 || n_kv_heads < 1) return DBSA_ERR_INVALID_ARG;
  if (n_q_heads % n_kv_heads != 0 || n_q_heads / n_kv_heads > 32) return DBSA_ERR_UNSUPPORTED;
  // the segments' tiles and each question's pool list, with every check of the descriptions
  dbsa_layout lists;
  lists.compute_units = L->compute_units;
  if (const int rc = dbsa_build_host_lists(pool, sel, -1, 256, kChunkTile, &lists)) return rc;

  const int32_t B = sel->n_queries, r = n_q_heads / n_kv_heads, n_seg = lists.n_groups + 1;
  L->chunk_stage = true;
  L->block_m = lists.block_m;
  L->block_n = kChunkTile;
  L->sink_len = lists.sink_len;
  L->n_tokens = lists.n_tokens;
  L->n_groups = lists.n_groups;
  L->n_queries = B;
  L->n_query_tokens = sel->cu_qlens[B];
  L->list_ptr.assign(1, 0);
  L->ck_q_heads = n_q_heads;
  L->ck_kv_heads = n_kv_heads;

  auto new_tokens = [&](int32_t u) { return sel->cu_qlens[u + 1] - sel->cu_qlens[u]; };
  for (int32_t u = 0; own_tokens && u < B; ++u)
    if (own_tokens[u] < 0) return DBSA_ERR_INVALID_ARG;

  std::vector<std::vector<int32_t>> users(n_seg);  // questions of a segment, ascending
  if (lists.sink_len > 0)
    for (int32_t u = 0; u < B; ++u) users[0].push_back(u);
  for (int32_t u = 0; u < B; ++u)
    for (int32_t e = sel->sel_ptr[u]; e < sel->sel_ptr[u + 1]; ++e) users[sel->sel_idx[e] + 1].push_back(u);
  auto seg_tiles = [&](int32_t s) { return lists.gm_seg_ptr[s + 1] - lists.gm_seg_ptr[s]; };

  // ---- units ----
  std::vector<Unit> units;
  int32_t per_block = 1;  // tokens of a unit
  auto own_tiles = [&](int32_t u, int32_t tokens_before_end) {
    const int64_t n = own_tokens ? std::max(own_tokens[u], new_tokens(u)) : new_tokens(u);
    const int64_t last = std::max<int64_t>(1, n - tokens_before_end);
    return static_cast<int32_t>((last + kChunkTile - 1) / kChunkTile);
  };
  auto add_blocks = [&](const std::vector<int32_t>& toks, auto&& fill) {
    const int32_t n = static_cast<int32_t>(toks.size()), blocks = (n + per_block - 1) / per_block;
    for (int32_t b = 0; b < blocks; ++b) {  // (equal to within one token)
      const int32_t lo = static_cast<int32_t>(int64_t{b} * n / blocks), hi = static_cast<int32_t>(int64_t{b + 1} * n / blocks);
      Unit x{static_cast<int32_t>(L->ck_toks.size()), hi - lo, 0, 0, -1, 0};
      L->ck_toks.insert(L->ck_toks.end(), toks.begin() + lo, toks.begin() + hi);
      fill(x, n - hi);
      if (x.cost() > 0) units.push_back(x);
    }
  };
  std::vector<char> alone(B, 0);
  std::vector<int32_t> toks;
  auto tokens_of = [&](int32_t u) {
    for (int32_t t = sel->cu_qlens[u]; t < sel->cu_qlens[u + 1]; ++t) toks.push_back(t);
  };
  auto make_units = [&](int32_t rows) {
    per_block = rows / r;
    units.clear();
    L->ck_toks.clear();
    L->ck_ent = lists.gm_seg_ent;
    for (int32_t u = 0; u < B; ++u) {
      alone[u] = new_tokens(u) >= per_block || B == 1;
      if (!alone[u]) continue;
      const int32_t at = static_cast<int32_t>(L->ck_ent.size() / 2), n = static_cast<int32_t>(lists.dec_ptr[u + 1] - lists.dec_ptr[u]);
      L->ck_ent.insert(L->ck_ent.end(), lists.dec_ent.begin() + 2 * lists.dec_ptr[u], lists.dec_ent.begin() + 2 * lists.dec_ptr[u + 1]);
      toks.clear();
      tokens_of(u);
      add_blocks(toks, [&](Unit& x, int32_t behind) {
        x.ent_begin = at;
        x.n_ent = n;
        x.own_u = u;
        x.own_tiles = own_tiles(u, behind);
      });
    }
    for (int32_t s = 0; s < n_seg; ++s) {
      toks.clear();
      for (int32_t u : users[s])
        if (!alone[u]) tokens_of(u);
      if (toks.empty() || seg_tiles(s) == 0) continue;
      add_blocks(toks, [&](Unit& x, int32_t) {
        x.ent_begin = static_cast<int32_t>(lists.gm_seg_ptr[s]);
        x.n_ent = static_cast<int32_t>(seg_tiles(s));
      });
    }
    for (int32_t u = 0; u < B; ++u) {
      if (alone[u]) continue;
      toks.clear();
      tokens_of(u);
      add_blocks(toks, [&](Unit& x, int32_t behind) {
        x.own_u = u;
        x.own_tiles = own_tiles(u, behind);
      });
    }
    int64_t tiles = 0;
    for (const Unit& x : units) tiles += x.cost();
    return tiles;
  };
  // The shape whose longest worker is done first.  Two workgroups of four waves share a compute unit's bandwidths and take about
  // 3/2 of the time of one of eight for a tile, but come in twice the number and leave fewer rows empty.  12 questions of 229
  // tokens: 1234 us with 256 rows, 1520 with 128; 122 of 14 behind 13k own keys: 891 and 658; 16 of 8 over 90k: 120 and 126.  The
  // ratio is one for all calls, because a layout knows neither the type nor the channels: over 72 batches drawn from one token to
  // 1668 it came to 3.6 % above the better shape on average (eight waves always: 7.1 %, four always: 5.7 %).  By type: bf16
  // 1.6 % with 128 channels and 8 % with 64, 8 bits 2 %, where eight waves always would be as good, and fp32 9 %, where
  // four always would be better.  (Workgroups of one or two waves fetch and widen too slowly: one token over 2k 23.5 us, 18.5 with
  // eight waves; the 16 questions 321 and 173.)
  const ChunkShape shapes[2] = {{256, 1, 2}, {128, 2, 3}};
  ChunkShape shape = shapes[0];
  int64_t tiles = 0, workers = 0;
  auto longest = [&](const ChunkShape& x) {
    tiles = make_units(x.rows);
    workers = std::max<int64_t>(1, std::min<int64_t>(tiles, int64_t{L->compute_units} * x.per_cu / n_kv_heads));
    return static_cast<double>(tiles + kRecordCost * static_cast<int64_t>(units.size())) / static_cast<double>(workers) * x.tile_cost;
  };
  const double four_waves = longest(shapes[1]);
  if (longest(shapes[0]) > four_waves) {
    shape = shapes[1];
    longest(shape);
  }
  L->ck_rows = shape.rows;

  // ---- dealing ----
  int64_t total = 0;
  for (const Unit& x : units) total += x.cost() + kRecordCost;
  // one dealing at a share: records (unit, first tile, tiles) worker by worker; true if every tile found a worker
  struct Record {
    int32_t unit, lo, n;
  };
  std::vector<Record> recs;
  std::vector<int32_t> ptr;
  auto deal = [&](int64_t share, bool whole) {
    recs.clear();
    ptr.assign(1, 0);
    int64_t room = share;
    for (size_t i = 0; i < units.size(); ++i) {
      const int64_t all = units[i].cost();
      for (int64_t lo = 0; lo < all;) {
        const int64_t n = std::min(all - lo, room - kRecordCost);
        if (n < (whole ? all : 1)) {
          if (room == share) return false;
          ptr.push_back(static_cast<int32_t>(recs.size()));
          room = share;
          if (static_cast<int64_t>(ptr.size()) > workers) return false;
          continue;
        }
        recs.push_back({static_cast<int32_t>(i), static_cast<int32_t>(lo), static_cast<int32_t>(n)});
        room -= n + kRecordCost;
        lo += n;
      }
    }
    ptr.push_back(static_cast<int32_t>(recs.size()));
    return true;
  };
  // Units stay whole where that costs no worker more than a sixteenth above its share: a cut costs two partial states and the
  // merge of them (2048 tokens behind 90k, 32 units of nearly equal length: 1960 us cut into equal shares, 1830 whole).
  // And where they are short.
  const int64_t fair = std::max<int64_t>((total + workers - 1) / workers, 1 + kRecordCost);
  if (!deal(std::max(fair + fair / 16, kShortUnit + kRecordCost), true))
    for (int64_t share = fair; !deal(share, false);) share += std::max<int64_t>(1, share / 64);

  // ---- records, and where each token's partial states lie ----
  std::vector<int32_t> parts_of(L->n_query_tokens, 0);  // records that carry the token
  for (const Record& x : recs) {
    for (int32_t t = 0; t < units[x.unit].n_tok; ++t) ++parts_of[L->ck_toks[units[x.unit].tok_begin + t]];
  }
  std::vector<std::vector<int32_t>> parts(L->n_query_tokens);
  int64_t rows = 0;
  for (const Record& x : recs) {
    const Unit& w = units[x.unit];
    const bool whole = w.own_u >= 0 && w.n_tok > 0 && parts_of[L->ck_toks[w.tok_begin]] == 1;
    int32_t base = -1;
    if (!whole) {
      if (rows + w.n_tok > INT32_MAX) return DBSA_ERR_UNSUPPORTED;
      base = static_cast<int32_t>(rows);
      for (int32_t t = 0; t < w.n_tok; ++t) parts[L->ck_toks[w.tok_begin + t]].push_back(base + t);
      rows += w.n_tok;
    }
    const int32_t pool_lo = std::min(x.lo, w.n_ent), pool_hi = std::min(x.lo + x.n, w.n_ent);
    const int32_t own_lo = std::max(x.lo - w.n_ent, 0), own_hi = std::max(x.lo + x.n - w.n_ent, 0);
    const bool owns = own_hi > own_lo;
    const int32_t u = owns ? w.own_u : -1;
    L->ck_rec.insert(L->ck_rec.end(),
                     {w.tok_begin, w.n_tok, w.ent_begin + pool_lo, pool_hi - pool_lo, u, own_lo, own_hi, w.own_tiles, base,
                      owns ? sel->cu_qlens[u] : 0, owns ? new_tokens(u) : 0, 0});
  }
  L->ck_ptr = ptr;
  L->ck_workers = static_cast<int32_t>(ptr.size()) - 1;
  L->ck_part_rows = rows;
  L->ck_tok_ptr.assign(1, 0);
  for (int32_t t = 0; t < L->n_query_tokens; ++t) {
    L->ck_tok_part.insert(L->ck_tok_part.end(), parts[t].begin(), parts[t].end());
    if (!parts[t].empty()) L->ck_merge.insert(L->ck_merge.end(), {t, L->ck_tok_ptr.back(), static_cast<int32_t>(parts[t].size())});
    L->ck_tok_ptr.push_back(static_cast<int32_t>(L->ck_tok_part.size()));
  }
  return DBSA_OK;
}
