// attention_span.h -- the launcher of attention over parts of the requests' keys.
#pragma once

#include "mx_kernels.h"
#include "span.h"

namespace mx {

struct SpanParams {
  AttnParams a;  // reqs, items, split_pages and decode_only unused
  const SpanItem* items;
  const int32_t* tokens;
  const SpanToken* merge_tokens;
  const SpanSource* sources;
  int32_t window, sinks;
  int32_t n_items;    // of each KV head
  int32_t heads;      // of a group (span_block)
  uint32_t group_inv; // 2^32 / group, rounded up (group > 1)
};

// The items of every head, then the merge of n_merge tokens whose rows have up to
// most_parts partials.  meta, where given, holds the metadata (the pointers into it are
// offsets there), handed over with the kernels' arguments.
hipError_t launch_span_attn(const SpanParams& p, const InlineMeta* meta, bool tiles, int n_merge,
                            int most_parts, int head_dim, hipStream_t stream);

}  // namespace mx
