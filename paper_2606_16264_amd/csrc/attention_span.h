// attention_span.h -- the launcher of attention over parts of the requests' keys.
#pragma once

#include "mx_kernels.h"
#include "span.h"

namespace mx {

struct SpanParams {
  AttnParams a;  // reqs, items, split_pages and decode_only unused
  const SpanRows* rows;
  const SpanItem* items;
  const int32_t* tokens;
  int32_t window, sinks;
};

// The items, then the merge of `n_merge` tokens (wide: by a workgroup for each q head).
hipError_t launch_span_attn(const SpanParams& p, int n_items, bool tiles, const SpanToken* merge,
                            int n_merge, bool wide, const SpanMerge* merges,
                            const SpanSource* sources, int head_dim, hipStream_t stream);

}  // namespace mx
