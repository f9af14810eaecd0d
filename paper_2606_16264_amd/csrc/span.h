// span.h -- attention over parts of the requests' keys: what the host planner hands to
// the kernels of attention_span.hip.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define MX_SPAN_FN __host__ __device__ __forceinline__
#else
#define MX_SPAN_FN inline
#endif

namespace mx {

constexpr int kSpanTileRows = 128;   // four waves x two blocks of 16 rows
constexpr int kSpanStreamRows = 16;

// Rows that share their keys, of every KV head: row r is token r / group of the rows'
// tokens and q head (KV head) * group + r % group.  The keys' pages stand in a table of
// their own, without the pages between sink_pages and sink_pages + skip of the request:
// entry t is the request's page t, or t + skip from sink_pages on.
//
// With n_split items over the keys of the same rows, or parts of other records for them,
// row r leaves split s of KV head g at partial part + (g * n_split + s) * n_rows + r.
struct SpanRows {
  int32_t tok;         // batch row of token 0; list: the offset of the tokens' list
  int32_t n_rows;      // tokens * group
  int32_t pos;         // position of token 0; list: of every token
  int32_t list;        // the tokens' batch rows stand in a list of their own
  int32_t pages, entries;  // the page table: its offset in the flat page array, its length
  int32_t sink_pages, skip;
  int32_t n_split;
  int32_t part;        // -1: the rows go to the output
};

// The pages of some rows: page0 .. page1 - 1, counted without the `skip` entries of the table
// from sink_pages on that none of the rows sees.
struct SpanPages {
  int32_t skip, page0, page1;
};
// All that tokens tok0 .. tok1 of a record see.
inline SpanPages span_seen(const SpanRows& r, int tok0, int tok1, int window) {
  if (r.list) return SpanPages{0, 0, r.entries};
  const int pos0 = r.pos + tok0, pos1 = r.pos + tok1;
  const int low = pos0 < window ? 0 : (pos0 - window + 1) >> 4;  // the first page of the window
  // (of the request's pages; the table has left out r.skip of them already)
  const int cut = low - r.sink_pages - r.skip, skip = cut > 0 ? cut : 0;
  const int last = (pos1 >> 4) < r.sink_pages ? (pos1 >> 4) : (pos1 >> 4) - r.skip;
  return SpanPages{skip, 0, (last + 1 < r.entries ? last + 1 : r.entries) - skip};
}
// Split `split` of `n_split`, in whole chunks of two pages.  (Empty where there are fewer
// chunks than splits: the rows' partials are zeros.)
inline SpanPages span_split(SpanPages s, int split, int n_split) {
  if (n_split == 1) return s;
  const int chunks = (s.page1 + 1) >> 1;
  const int per = chunks / n_split, more = chunks - per * n_split;  // the first `more` take one more
  const int first = split * per + (split < more ? split : more);
  const int end = 2 * (first + per + (split < more ? 1 : 0));
  return SpanPages{s.skip, 2 * first, end < s.page1 ? end : s.page1};
}

// A work item, of each KV head a workgroup: `n_rows` rows of a record, over some of its pages.
//   kind 0 (stream): up to kSpanStreamRows rows
//   kind 1 (tile):   up to kSpanTileRows rows
// All that a workgroup has to know before its first loads stands here: each record read on the
// way to them costs it most of a microsecond.
struct SpanItem {
  int32_t tok;          // batch row, or place in the list, of the first row's token
  int32_t rest;         // the first row's place among the group rows of its token
  int32_t pos;          // position of that token; list: of every token
  int32_t list;
  int32_t pages, sink_pages;
  int32_t skip_table, skip_real;  // entries and pages left out from sink_pages on
  int32_t page0, page1;           // counted without them
  int32_t part, kvh_stride;       // partial of the first row of KV head 0 (-1: output), of the next head
  int32_t kind, n_rows;
  int32_t pad[2];
};

// The item and KV head of a workgroup.  The heads go by groups of `heads`, of each group all
// items, each item's heads one after the other.  Workgroup b runs on die b % 8, each die with
// an L2 of its own: in groups of eight heads (or where their number is a multiple of eight)
// the items of a head run on one die, and in groups of eight also one after the other, so
// that a prompt's tiles find the keys of their neighbours there.
struct SpanBlock {
  int item, kvh;
};
MX_SPAN_FN SpanBlock span_block(int b, int n_items, int nkv, int heads) {
  const int full = heads * n_items, group = b / full, at = b - group * full;
  const int left = nkv - heads * group, here = left < heads ? left : heads;
  return SpanBlock{at / here, heads * group + at % here};
}

// Partials of a request's tokens: split s of KV head g, row i of its token t's group at
// base + g * kvh_stride + s * split_stride + t * group + i.
struct SpanSource {
  int32_t base, kvh_stride, split_stride, n_split;
};
// A token to be merged: its batch row, the sources of its request, its place there.
struct SpanToken {
  int32_t tok, src, n_src, at;
};

}  // namespace mx
