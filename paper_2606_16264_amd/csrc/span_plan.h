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

struct SpanPlan {
  int group = 1, nkv = 1;
  int window = INT32_MAX, sinks = 0;
  struct Table {  // entries first .. first + n - 1 of a request's page table
    const int32_t* pages;
    int n;
  };
  std::vector<SpanRows> rows;
  std::vector<Table> tables;  // whose entries follow each other in the flat page array
  std::vector<int32_t> tokens;
  std::vector<SpanItem> items;
  std::vector<SpanSource> sources;
  std::vector<SpanMerge> merges;
  std::vector<SpanToken> merge_tokens;
  int64_t n_pages = 0, n_parts = 0;
  int most_parts = 0;  // partials of a row
  bool has_tiles = false;

  int add_table(const int32_t* pages, int n) {
    const int at = (int)n_pages;
    tables.push_back(Table{pages, n});
    n_pages += n;
    return at;
  }
};

namespace plan {

constexpr int kXcds = 8;           // workgroup b runs on die b % 8
constexpr int64_t kSlots = 512;    // workgroups that the chip holds at once
constexpr int kMinSplitPages = 16; // of a stream, and of a tile (below)
constexpr int kMinTilePages = 32;
constexpr int kExtraTiles = 1024;  // items that splitting tiles adds to a call, at most

// Rows with the pages that they take, before they are cut into items.
struct Part {
  int rows;        // SpanRows index
  bool stream;
  bool partial;    // the rows have other parts
  int source;      // of a partial part: its SpanSource
};

// The pages of rows row0 .. row0 + n - 1, counted as in SpanItem.
struct Range {
  int skip, end;
};
inline Range range_of(const SpanPlan& p, const SpanRows& r, int entries, int row0, int n) {
  if (r.list) return {0, entries};
  const int pos0 = r.pos + row0 / p.group, pos1 = r.pos + (row0 + n - 1) / p.group;
  const int first = (int)(std::max<int64_t>(0, (int64_t)pos0 - p.window + 1) / 16);
  // (of the request's pages; the table has left out r.skip of them already)
  const int skip = std::max(0, first - r.sink_pages - r.skip);
  const int last = pos1 / 16 < r.sink_pages ? pos1 / 16 : pos1 / 16 - r.skip;
  return {skip, std::min(entries, last + 1) - skip};
}

}  // namespace plan

// Cuts the parts into items and orders them.  entries[i]: table entries of rows record i.
inline void plan_items(SpanPlan& p, const std::vector<plan::Part>& parts,
                       const std::vector<int>& entries) {
  using namespace plan;
  // how much there is to do: pages of streams, and of tiles
  int64_t stream_pages = 0, tile_pages = 0;
  for (const Part& part : parts) {
    const SpanRows& r = p.rows[part.rows];
    const int step = part.stream ? 16 : kSpanTileRows;
    for (int row = 0; row < r.n_rows; row += step) {
      const int64_t n = range_of(p, r, entries[part.rows], row, std::min(step, r.n_rows - row)).end;
      (part.stream ? stream_pages : tile_pages) += n * p.nkv;
    }
  }
  const int stream_split = (int)std::max<int64_t>(kMinSplitPages, (stream_pages + 1023) / 1024 + 1) & ~1;
  const int tile_split = (int)std::max<int64_t>(kMinTilePages, (tile_pages + kSlots - 1) / kSlots + 1) & ~1;
  std::vector<SpanItem> list[2];
  int64_t extra = kExtraTiles;
  for (const Part& part : parts) {
    const SpanRows& r = p.rows[part.rows];
    const int step = part.stream ? 16 : kSpanTileRows;
    // splits: as many for every item of the part, so that a row's partials are found
    int most = 0;
    for (int row = 0; row < r.n_rows; row += step)
      most = std::max(most, range_of(p, r, entries[part.rows], row, std::min(step, r.n_rows - row)).end);
    int n_split = std::max(1, most / (part.stream ? stream_split : tile_split));
    if (!part.stream) {
      const int64_t tiles = (int64_t)((r.n_rows + step - 1) / step) * p.nkv;
      n_split = (int)std::min<int64_t>(n_split, 1 + extra / tiles);
      extra -= (n_split - 1) * tiles;
    }
    const bool partial = part.partial || n_split > 1;
    if (partial) {
      SpanSource& s = p.sources[part.source];
      s.base = (int32_t)p.n_parts;
      s.split_stride = r.n_rows;
      s.kvh_stride = n_split * r.n_rows;
      s.n_split = n_split;
    }
    for (int g = 0; g < p.nkv; g++)
      for (int row = 0; row < r.n_rows; row += step) {
        const int n = std::min(step, r.n_rows - row);
        const Range range = range_of(p, r, entries[part.rows], row, n);
        const int chunks = (range.end + 1) / 2;
        for (int s = 0; s < n_split; s++) {
          // (empty where a tile has fewer chunks than splits: its rows' partials are zeros)
          const int page0 = 2 * (int)((int64_t)chunks * s / n_split);
          const int page1 = std::min(range.end, 2 * (int)((int64_t)chunks * (s + 1) / n_split));
          const int64_t part_at = partial ? p.n_parts + ((int64_t)g * n_split + s) * r.n_rows + row : -1;
          list[part.stream ? 0 : 1].push_back(SpanItem{part.rows, (int16_t)g, (int8_t)(part.stream ? 0 : 1),
                                                       (uint8_t)n, row, page0, page1, range.skip,
                                                       (int32_t)part_at, 0});
        }
      }
    if (partial) p.n_parts += (int64_t)p.nkv * n_split * r.n_rows;
  }
  auto longer = [](const SpanItem& a, const SpanItem& b) {
    return a.page_end - a.page0 > b.page_end - b.page0;
  };
  for (auto& l : list) std::stable_sort(l.begin(), l.end(), longer);
  p.has_tiles = !list[1].empty();
  p.items = std::move(list[1]);
  p.items.insert(p.items.end(), list[0].begin(), list[0].end());
}

// The merges of the requests' tokens: of each request its sources, whose bases count from
// its first token.
struct RequestSources {
  int tok, n_new;
  std::vector<std::pair<int, int>> from;  // (source, the request's first token in it)
};
inline void plan_merges(SpanPlan& p, const std::vector<RequestSources>& reqs) {
  std::vector<SpanSource> out;
  for (const RequestSources& q : reqs) {
    int n = 0;
    SpanMerge m{q.tok, (int)out.size(), 0, 0};
    for (const auto& f : q.from) {
      SpanSource s = p.sources[f.first];
      if (s.n_split == 0) continue;  // the rows went to the output
      s.base += f.second * p.group;
      n += s.n_split;
      out.push_back(s);
      m.n_src++;
    }
    if (m.n_src == 0) continue;
    p.most_parts = std::max(p.most_parts, n);
    for (int i = 0; i < q.n_new; i++) p.merge_tokens.push_back(SpanToken{q.tok + i, (int)p.merges.size()});
    p.merges.push_back(m);
  }
  p.sources = std::move(out);
}

inline void plan_window(const mx_batch* b, const mx_attn_shape* s, int window, int sinks, SpanPlan& p) {
  p.nkv = s->n_kv_heads;
  p.group = s->n_q_heads / s->n_kv_heads;
  p.window = window;
  p.sinks = sinks;
  std::vector<plan::Part> parts;
  std::vector<int> entries;
  std::vector<RequestSources> reqs;
  int tok = 0;
  for (int r = 0; r < b->num_reqs; r++) {
    const mx_request& q = b->reqs[r];
    const SeenPages seen = seen_pages(q.ctx_len, q.n_new, window, sinks);
    const int at = p.add_table(q.pages, seen.sink_pages);
    p.add_table(q.pages + seen.sink_pages + seen.skip, seen.entries() - seen.sink_pages);
    p.rows.push_back(SpanRows{tok, q.n_new * p.group, q.ctx_len, 0, at, seen.sink_pages, seen.skip, 0});
    entries.push_back(seen.entries());
    parts.push_back(plan::Part{r, q.n_new == 1, false, r});
    reqs.push_back(RequestSources{tok, q.n_new, {{r, 0}}});
    tok += q.n_new;
  }
  p.sources.assign(b->num_reqs, SpanSource{0, 0, 0, 0});
  plan_items(p, parts, entries);
  plan_merges(p, reqs);
}

// Shared runs: start[r] of a request's pages belong to runs; first[i] is the first page of
// run i in its members' tables.
inline void plan_shared(const mx_batch* b, const mx_attn_shape* s, int num_runs,
                        const mx_shared_run* runs, SpanPlan& p) {
  p.nkv = s->n_kv_heads;
  p.group = s->n_q_heads / s->n_kv_heads;
  const int R = b->num_reqs;
  std::vector<plan::Part> parts;
  std::vector<int> entries;
  std::vector<RequestSources> reqs(R);
  std::vector<int> start(R, 0), own(R, 0);  // pages before: in runs so far; not the request's own
  // A prompt whose rows fill tiles by themselves takes its shared keys with its own: the
  // rows that would be saved, times the keys, against partials for all of its rows.
  std::vector<char> whole(R, 0);
  for (int i = 0; i < num_runs; i++)
    for (int r = runs[i].first_req; r < runs[i].first_req + runs[i].num_reqs; r++) start[r] += runs[i].n_pages;
  int tok = 0;
  for (int r = 0; r < R; r++) {
    const mx_request& q = b->reqs[r];
    const int64_t rows = (int64_t)q.n_new * p.group;
    const int64_t spare = (rows + kSpanTileRows - 1) / kSpanTileRows * kSpanTileRows - rows;
    whole[r] = q.n_new > 1 && spare * start[r] * 16 <= rows * 1024;
    reqs[r] = RequestSources{tok, q.n_new, {}};
    tok += q.n_new;
    start[r] = 0;
  }
  // how many requests take part in each run; a run of one is that request's own
  for (int i = 0; i < num_runs; i++) {
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
    const int rec = (int)p.rows.size(), src = (int)p.sources.size();
    p.sources.push_back(SpanSource{0, 0, 0, 0});
    const int list = (int)p.tokens.size();
    int at = 0;
    for (int r = run.first_req; r < end; r++) {
      if (whole[r]) continue;
      reqs[r].from.push_back({src, at});
      for (int t = 0; t < b->reqs[r].n_new; t++) p.tokens.push_back(reqs[r].tok + t);
      at += b->reqs[r].n_new;
      own[r] = start[r];
    }
    const int pages = p.add_table(b->reqs[leader].pages + first, run.n_pages);
    p.rows.push_back(SpanRows{list, n_tok * p.group, INT32_MAX / 2, 1, pages, 0, 0, 0});
    entries.push_back(run.n_pages);
    parts.push_back(plan::Part{rec, n_tok * p.group <= 16, true, src});
  }
  for (int r = 0; r < R; r++) {
    const mx_request& q = b->reqs[r];
    const int end = (q.ctx_len + q.n_new - 1) / 16 + 1;
    const int rec = (int)p.rows.size(), src = (int)p.sources.size();
    p.sources.push_back(SpanSource{0, 0, 0, 0});
    const int pages = p.add_table(q.pages + own[r], end - own[r]);
    p.rows.push_back(SpanRows{reqs[r].tok, q.n_new * p.group, q.ctx_len, 0, pages, 0, own[r], 0});
    entries.push_back(end - own[r]);
    parts.push_back(plan::Part{rec, q.n_new == 1, own[r] > 0, src});
    reqs[r].from.push_back({src, 0});
  }
  plan_items(p, parts, entries);
  plan_merges(p, reqs);
}

}  // namespace mx
