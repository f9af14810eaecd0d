// span_plan.h -- the host's plan of an attention over parts of the requests' keys
// (span.h): which pages an item takes for which rows, in what order the items run, and
// where the partial results of a row lie.
#pragma once

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <vector>

#include "mx.h"
#include "span.h"

namespace mx {

// What new tokens at positions ctx .. ctx + n - 1 see of their request, as pages: 0 ..
// sink_pages - 1 and sink_pages + skip .. end - 1.
struct SeenPages {
  int sink_pages, skip, end;
  int entries() const { return end - skip; }
};
inline SeenPages seen_pages(int ctx, int n, int window, int sinks) {
  SeenPages s;
  s.end = (int)(((int64_t)ctx + n - 1) / 16 + 1);
  s.sink_pages = std::min((int)(((int64_t)sinks + 15) / 16), s.end);
  const int first = (int)(std::max<int64_t>(0, (int64_t)ctx - window + 1) / 16);
  s.skip = std::max(0, first - s.sink_pages);
  return s;
}

// Joining the parts of a row costs a launch, partials written and read: all runs of a call are
// left to their requests where less than this, in sum, would be read once instead of several
// times.  (Over batches drawn at random a limit of 24 MB takes 0.4 to 1.3% more than one of
// 64.  Once a call is above it all of its runs are joined, the short ones too: not measured
// against joining some of them.)
constexpr int64_t kMinSharedBytes = 64 << 20;

struct SpanPlan {
  int64_t min_shared_bytes = kMinSharedBytes;
  int group = 1, nkv = 1;
  int64_t page_bytes = 0;  // keys and values of one head
  int window = INT32_MAX, sinks = 0;
  std::vector<SpanRows> rows;
  std::vector<int32_t> pages;  // the records' page tables
  std::vector<int32_t> tokens;
  std::vector<SpanItem> items;
  std::vector<SpanSource> sources;
  std::vector<SpanToken> merge_tokens;
  int64_t n_parts = 0;  // (numbered in 32 bits: the caller refuses a plan with more)
  int most_parts = 0;  // partials of a row
  bool has_tiles = false;
  int heads = 1;  // of a group of span_block

  int64_t blocks() const { return (int64_t)items.size() * nkv; }
  int add_table(const int32_t* ids, int n) {
    const int at = (int)pages.size();
    pages.insert(pages.end(), ids, ids + n);
    return at;
  }
};

namespace plan {

// (Both sides of each, over batches drawn at random.  Splits of streams of 16 pages instead of
// 32: 1% more, the metadata of 4 decodes through 1500 keys on 32 heads no longer goes with the
// arguments and they take 25.2 us for 20.4; of 48: up to a quarter more for a few decodes.
// Whole streams of up to 32 pages only: 2% more; up to 128: nothing gained.  Whole tiles of up
// to 16 pages only: 250 tokens in three prompts behind a run take 24.1 for 20.6; up to 96:
// nothing.  Splits of tiles of 32 pages where they are alone: 1 to 3% more.)
constexpr int64_t kSlots = 512;      // workgroups that the chip holds at once
constexpr int kMinSplitPages = 32;   // of a stream's split
constexpr int kWholePages = 64;      // streams of up to that many are not split
constexpr int kWholeTilePages = 48;  // tiles of up to that many are not split
constexpr int kMinTilePages = 16;    // of a tile's split
constexpr int kLongTilePages = 128;  // a split that one more joining of partials hardly adds to
constexpr int kFullPages = 16;       // streams of so many for each workgroup fill the chip
constexpr int kExtraTiles = 1024;    // items that splitting tiles adds to a call, at most
constexpr int kMostSplits = 4096;

// A record's rows, before they are cut into items.
struct Part {
  bool stream;
  bool partial;  // its rows have other parts
};

// Whether a record's rows run as streams: a decode's, and so few that a stream holds them, which
// has four waves share the keys where a tile would have one wave with rows and three without:
// chunks of 2 to 4 tokens behind 2000 to 8000 keys take 11 to 15 us, as tiles 14 to 19, and 16
// of them on 32 KV heads 20 and 25.  17 to 64 rows of several tokens as streams of 16 would read
// their keys again for each: up to a quarter less where a few requests are alone, half more in
// other batches.  A lone token's group of more than 16 q heads does run so, as in mx_paged_attn:
// 64 decodes behind 8000 keys take 99 us with 20 q heads on a KV head and 183 with 64 on two, 96
// and 184 there, 2.7 and 2.9 TB/s of what they have to read; as tiles they were not measured.
inline bool is_stream(const SpanRows& r, int group) {
  return r.n_rows <= kSpanStreamRows || (!r.list && r.n_rows == group);
}

// The launch order, both kinds longest first.  Streams are bound by HBM, tiles by the matrix
// cores, and interleaved they share a CU; but all tiles have to start early enough to end
// with the rest, so they are dealt out over the first part of the list, the share of it that
// is left of the whole when one tile's time is taken off its end.  (1024 tokens beside 64
// decodes: 68 us, all tiles first 75; dealt evenly to the end those take 64, but 128 decodes
// of one document of 16384 tokens 136 for 110.)
struct Cost {
  SpanItem item;
  int64_t cost;
};
// (1.0: those 1024 tokens take 74 us, the tree as long; 2.4: 70, the tree 63 for 62.)
constexpr double kStreamPage = 1.6;  // time of a stream's page, in tile pages
inline void order_items(std::vector<Cost>& tiles, std::vector<Cost>& streams, int nkv,
                        std::vector<SpanItem>& out) {
  auto longer = [](const Cost& a, const Cost& b) { return a.cost > b.cost; };
  double sum[2] = {};
  std::vector<Cost>* list[2] = {&tiles, &streams};
  for (int k = 0; k < 2; k++) {
    if (!std::is_sorted(list[k]->begin(), list[k]->end(), longer))
      std::stable_sort(list[k]->begin(), list[k]->end(), longer);
    for (const Cost& c : *list[k]) sum[k] += c.cost * (k ? kStreamPage : 1.0);
  }
  const double all = sum[0] + sum[1];
  const double share = tiles.empty() ? 1.0 : 1.0 - tiles[0].cost * (double)kSlots / (all * nkv);
  out.reserve(tiles.size() + streams.size());
  size_t j = 0;
  double done[2] = {};
  for (size_t i = 0; i < tiles.size() || j < streams.size();) {
    const bool tile = i < tiles.size() && (j >= streams.size() || done[0] * share * all <= (done[0] + done[1]) * sum[0]);
    if (tile) done[0] += tiles[i].cost, out.push_back(tiles[i++].item);
    else done[1] += streams[j].cost * kStreamPage, out.push_back(streams[j++].item);
  }
}

}  // namespace plan

// Cuts the records' rows into items and orders them.
inline void plan_items(SpanPlan& p, const std::vector<plan::Part>& parts) {
  using namespace plan;
  auto seen = [&](const SpanRows& r, int row, int n) {
    return span_seen(r, row / p.group, (row + n - 1) / p.group, p.window).page1;
  };
  // how much there is to do, in pages of one head
  int64_t pages[2] = {};
  int longest = 0;
  for (size_t i = 0; i < parts.size(); i++) {
    const SpanRows& r = p.rows[i];
    const int tile = !parts[i].stream, step = tile ? kSpanTileRows : kSpanStreamRows;
    for (int row = 0; row < r.n_rows; row += step) {
      const int n = seen(r, row, std::min(step, r.n_rows - row));
      pages[tile] += n;
      if (!tile) longest = std::max(longest, n);
    }
  }
  // Streams run whole where that fills the chip about evenly, and where they are short: a
  // split costs the merge's launch, which is what a few dozen pages take.
  const auto even = [](int64_t n) { return (int)(n + 1) & ~1; };
  const int64_t share = pages[0] * p.nkv / kSlots;  // of a workgroup that the chip holds at once
  const bool whole = longest <= std::max<int64_t>(kWholePages, share + share / 4);
  const int stream_split = whole ? longest : even(std::max<int64_t>(kMinSplitPages, share / 2));
  // Tiles are split to as many as the chip holds at once, or one for each CU beside streams
  // that take a good part of the time.  (Alone for each CU only: a prompt of 7659 tokens on 4
  // heads takes 80 us for 58, 371 tokens in 12 prompts on 40 heads 86 for 61.  Beside streams
  // as many as fit: 1024 tokens of 64 q heads beside 64 decodes 72.6 for 68.1.)  Where the streams
  // fill the chip as well, with splits of 32 pages, so that there is less to join: 32 decodes
  // of one prompt of 2000 take 44.4 us, with splits of 16 46.2; a tree 62.0 and 65.1.  Where
  // they do not the longest tile is the time: 45 decodes below six runs 25 us, 33 with 32.
  const bool mixed = pages[0] * kStreamPage > pages[1] / 4;
  const int64_t slots = mixed ? kSlots / 2 : kSlots;
  const int min_tile = mixed && pages[0] * p.nkv >= kFullPages * kSlots ? 2 * kMinTilePages : kMinTilePages;
  const int tile_split = even(std::max<int64_t>(min_tile, (pages[1] * p.nkv + slots - 1) / slots));
  std::vector<Cost> list[2];
  int64_t extra = kExtraTiles;
  for (size_t i = 0; i < parts.size(); i++) {
    SpanRows& r = p.rows[i];
    const int tile = !parts[i].stream, step = tile ? kSpanTileRows : kSpanStreamRows;
    // as many splits for every item of the record
    int most = 0, n_split = 1;
    for (int row = 0; row < r.n_rows; row += step)
      most = std::max(most, seen(r, row, std::min(step, r.n_rows - row)));
    if (!tile) {
      n_split = std::max(1, (most + stream_split / 2) / std::max(1, stream_split));
    } else if (most > kWholeTilePages || parts[i].partial) {
      // (as many as leave no split shorter, but where they are long and there is room beside one
      // for each CU the nearest number: 243 decodes of one document of 11232 tokens on 64 q
      // heads take 144 us for 229; over drawn batches of 60 us and more 1% less, where splits
      // are short a tenth more for some)
      n_split = std::max(1, (most + (mixed && tile_split >= kLongTilePages ? tile_split / 2 : 0)) / tile_split);
      const int64_t tiles = (int64_t)((r.n_rows + step - 1) / step) * p.nkv;
      n_split = (int)std::min<int64_t>(n_split, 1 + extra / tiles);
      extra -= (n_split - 1) * tiles;
    }
    n_split = std::min(n_split, kMostSplits);
    r.n_split = n_split;
    r.part = -1;
    if (parts[i].partial || n_split > 1) {
      r.part = (int32_t)p.n_parts;
      p.n_parts += (int64_t)p.nkv * n_split * r.n_rows;
    }
    // (tiles that take the same keys follow each other)
    for (int s = 0; s < n_split; s++)
      for (int row = 0; row < r.n_rows; row += step) {
        const int n = std::min(step, r.n_rows - row), tok0 = row / p.group;
        const SpanPages all = span_seen(r, tok0, (row + n - 1) / p.group, p.window);
        const SpanPages pg = span_split(all, s, n_split);
        SpanItem it = {};
        it.tok = r.tok + tok0;
        it.rest = row - tok0 * p.group;
        it.list = r.list;
        it.pos = r.list ? r.pos : r.pos + tok0;
        it.pages = r.pages;
        it.sink_pages = r.sink_pages;
        it.skip_table = pg.skip;
        it.skip_real = pg.skip + r.skip;
        it.page0 = pg.page0;
        it.page1 = pg.page1;
        it.part = r.part < 0 ? -1 : (int32_t)(r.part + (int64_t)s * r.n_rows + row);
        it.kvh_stride = (int32_t)((int64_t)n_split * r.n_rows);
        it.kind = tile;
        it.n_rows = n;
        list[tile].push_back(Cost{it, std::max(1, all.page1 / n_split)});
      }
  }
  p.has_tiles = !list[1].empty();
  // (streams find nothing in L2, and long tiles of the last heads would start too late)
  p.heads = list[0].empty() ? std::min(p.nkv, 8) : p.nkv;
  order_items(list[1], list[0], p.nkv, p.items);
}

// The merges of the requests' tokens: of each request the records that its tokens are rows of,
// and its first token there.
struct RequestSources {
  int tok, n_new;
  std::vector<std::pair<int, int>> from;
};
inline void plan_merges(SpanPlan& p, const std::vector<RequestSources>& reqs) {
  for (const RequestSources& q : reqs) {
    const int src = (int)p.sources.size();
    int n = 0;
    for (const auto& f : q.from) {
      const SpanRows& r = p.rows[f.first];
      if (r.part < 0) continue;  // the rows went to the output
      n += r.n_split;
      p.sources.push_back(SpanSource{(int32_t)(r.part + (int64_t)f.second * p.group),
                                     (int32_t)((int64_t)r.n_split * r.n_rows), r.n_rows, r.n_split});
    }
    const int n_src = (int)p.sources.size() - src;
    if (n_src == 0) continue;
    p.most_parts = std::max(p.most_parts, n);
    for (int i = 0; i < q.n_new; i++) p.merge_tokens.push_back(SpanToken{q.tok + i, src, n_src, i});
  }
}

inline void plan_shape(const mx_attn_shape* s, SpanPlan& p) {
  p.nkv = s->n_kv_heads;
  p.group = s->n_q_heads / s->n_kv_heads;
  p.page_bytes = 16 * 2 * 2 * s->head_dim;
}

inline void plan_window(const mx_batch* b, const mx_attn_shape* s, int window, int sinks, SpanPlan& p) {
  plan_shape(s, p);
  p.window = window;
  p.sinks = sinks;
  std::vector<plan::Part> parts;
  std::vector<RequestSources> reqs;
  int tok = 0;
  for (int r = 0; r < b->num_reqs; r++) {
    const mx_request& q = b->reqs[r];
    const SeenPages seen = seen_pages(q.ctx_len, q.n_new, window, sinks);
    const int at = p.add_table(q.pages, seen.sink_pages);
    p.add_table(q.pages + seen.sink_pages + seen.skip, seen.entries() - seen.sink_pages);
    p.rows.push_back(SpanRows{tok, q.n_new * p.group, q.ctx_len, 0, at, seen.entries(), seen.sink_pages, seen.skip, 1, -1});
    parts.push_back(plan::Part{plan::is_stream(p.rows.back(), p.group), false});
    reqs.push_back(RequestSources{tok, q.n_new, {{r, 0}}});
    tok += q.n_new;
  }
  plan_items(p, parts);
  plan_merges(p, reqs);
}

// A prompt whose rows fill tiles by themselves takes its shared keys with its own: the rows
// that would be saved, times the keys, against partials for all of its rows.  (With 512: 1500
// tokens in 12 prompts about one document beside 24 decodes of it take 219 us for 215; with
// 8192: nothing gained.)
constexpr int64_t kWholePromptKeys = 2048;

inline void plan_shared(const mx_batch* b, const mx_attn_shape* s, int num_runs,
                        const mx_shared_run* runs, SpanPlan& p) {
  plan_shape(s, p);
  const int R = b->num_reqs;
  std::vector<plan::Part> parts;
  std::vector<RequestSources> reqs(R);
  std::vector<int> start(R, 0), own(R, 0);  // pages of the runs so far; of the runs that r takes part in
  std::vector<char> whole(R, 0);            // takes no part in runs from here on
  for (int i = 0; i < num_runs; i++)
    for (int r = runs[i].first_req; r < runs[i].first_req + runs[i].num_reqs; r++) start[r] += runs[i].n_pages;
  int tok = 0;
  for (int r = 0; r < R; r++) {
    const mx_request& q = b->reqs[r];
    const int64_t rows = (int64_t)q.n_new * p.group;
    const int64_t spare = (rows + kSpanTileRows - 1) / kSpanTileRows * kSpanTileRows - rows;
    whole[r] = q.n_new > 1 && spare * start[r] * 16 <= rows * kWholePromptKeys;
    reqs[r] = RequestSources{tok, q.n_new, {}};
    tok += q.n_new;
    start[r] = 0;
  }
  int64_t saved = 0;
  for (int i = 0; i < num_runs; i++) {
    int takers = 0;
    for (int r = runs[i].first_req; r < runs[i].first_req + runs[i].num_reqs; r++) takers += !whole[r];
    if (takers > 1) saved += (takers - 1) * (int64_t)runs[i].n_pages * p.nkv * p.page_bytes;
  }
  for (int i = 0; saved >= p.min_shared_bytes && i < num_runs; i++) {
    const mx_shared_run& run = runs[i];
    const int end = run.first_req + run.num_reqs;
    int takers = 0, n_tok = 0, leader = -1;
    for (int r = run.first_req; r < end; r++)
      if (!whole[r]) {
        if (leader < 0) leader = r;
        takers++;
        n_tok += b->reqs[r].n_new;
      }
    const int first = start[run.first_req];
    for (int r = run.first_req; r < end; r++) start[r] += run.n_pages;
    if (takers == 0) continue;
    if (takers == 1) {  // from here on the request's own
      whole[leader] = 1;
      continue;
    }
    const int rec = (int)p.rows.size(), list = (int)p.tokens.size();
    int at = 0;
    for (int r = run.first_req; r < end; r++) {
      if (whole[r]) continue;
      reqs[r].from.push_back({rec, at});
      for (int t = 0; t < b->reqs[r].n_new; t++) p.tokens.push_back(reqs[r].tok + t);
      at += b->reqs[r].n_new;
      own[r] = start[r];
    }
    const int pages = p.add_table(b->reqs[leader].pages + first, run.n_pages);
    // (a position behind every key)
    p.rows.push_back(SpanRows{list, n_tok * p.group, INT32_MAX - 16, 1, pages, run.n_pages, 0, 0, 1, -1});
    parts.push_back(plan::Part{plan::is_stream(p.rows.back(), p.group), true});
  }
  for (int r = 0; r < R; r++) {
    const mx_request& q = b->reqs[r];
    const int end = (q.ctx_len + q.n_new - 1) / 16 + 1;
    reqs[r].from.push_back({(int)p.rows.size(), 0});
    const int pages = p.add_table(q.pages + own[r], end - own[r]);
    p.rows.push_back(SpanRows{reqs[r].tok, q.n_new * p.group, q.ctx_len, 0, pages, end - own[r], 0, own[r], 1, -1});
    parts.push_back(plan::Part{plan::is_stream(p.rows.back(), p.group), own[r] > 0});
  }
  plan_items(p, parts);
  plan_merges(p, reqs);
}

}  // namespace mx
