// span.h -- attention over parts of the requests' keys: what the host planner hands to
// the kernels of attention_span.hip.
#pragma once

#include <stdint.h>

namespace mx {

constexpr int kSpanTileRows = 128;  // four waves x two blocks of 16 rows

// Rows that share their keys, of every KV head: row r is token r / group of the rows'
// tokens and q head (KV head) * group + r % group.  The keys' pages stand in a table of
// their own, without the pages between sink_pages and sink_pages + skip of the request:
// entry t is the request's page t, or t + skip from sink_pages on.
struct SpanRows {
  int32_t tok;         // batch row of token 0; list: the offset of the tokens' list
  int32_t n_rows;      // tokens * group
  int32_t pos;         // position of token 0; list: of every token
  int32_t list;        // the tokens' batch rows stand in a list of their own
  int32_t pages;       // offset of the page table in the flat page array
  int32_t sink_pages, skip;
  int32_t pad;
};

// A work item: `n_rows` rows from row0 on, one KV head, over the pages page0 .. page_end - 1
// counted without the `skip` table entries from sink_pages on (pages that none of the
// item's rows sees).
//   kind 0 (stream): up to 16 rows of one position
//   kind 1 (tile):   up to kSpanTileRows rows
struct SpanItem {
  int32_t rows;
  int16_t kvh;
  int8_t kind;
  uint8_t n_rows;
  int32_t row0, page0, page_end, skip;
  int32_t part;  // partial of the item's first row, -1: the rows' output
  int32_t pad;
};

// Where partial results of a token's q heads lie: split s of KV head g, row i of the token's
// group at base + g * kvh_stride + s * split_stride + i.  (base: of a request's first token,
// `group` further for every next one)
struct SpanSource {
  int32_t base, kvh_stride, split_stride, n_split;
};
// A request whose tokens have partials: sources src .. src + n_src - 1.
struct SpanMerge {
  int32_t tok, src, n_src, pad;
};
struct SpanToken {  // a token to be merged
  int32_t tok, merge;
};

}  // namespace mx
