// What the host plans for batches of attention over parts of the keys (span_plan.h), as
// numbers: reads batches, prints a line of each.
//   in:  nq nkv head_dim min_shared_bytes (-1: the library's) window (0: shared runs) sinks,
//        requests, and of each n_new ctx_len n_pages ids, runs, and of each its three numbers
//   out: records of runs, tokens in them, and the sizes of the plan's arrays: items, page ids,
//        listed tokens, merged tokens, sources, partial rows
#include <cstdio>
#include <iostream>

#include "span_plan.h"

using namespace mx;

int main() {
  int nq, nkv, d, window, sinks, n_reqs, n_runs;
  int64_t least;
  while (std::cin >> nq >> nkv >> d >> least >> window >> sinks >> n_reqs) {
    std::vector<mx_request> reqs(n_reqs);
    std::vector<std::vector<int32_t>> pages(n_reqs);
    for (int r = 0; r < n_reqs; r++) {
      mx_request& q = reqs[r];
      std::cin >> q.n_new >> q.ctx_len >> q.n_pages;
      q.phase = q.n_new == 1 && q.ctx_len > 0 ? MX_DECODE : MX_PREFILL;
      pages[r].resize(q.n_pages);
      for (int32_t& id : pages[r]) std::cin >> id;
      q.pages = pages[r].data();
    }
    std::cin >> n_runs;
    std::vector<mx_shared_run> runs(n_runs);
    for (mx_shared_run& x : runs) std::cin >> x.first_req >> x.num_reqs >> x.n_pages;
    const mx_batch b{n_reqs, reqs.data()};
    const mx_attn_shape s{nq, nkv, d, 16, INT32_MAX, 0.f};
    SpanPlan p;
    if (least >= 0) p.min_shared_bytes = least;
    if (window > 0) plan_window(&b, &s, window, sinks, p);
    else plan_shared(&b, &s, n_runs, runs.data(), p);
    int lists = 0, in_lists = 0;
    for (const SpanRows& r : p.rows)
      if (r.list) lists++, in_lists += r.n_rows / p.group;
    printf("%d %d %zu %zu %zu %zu %zu %lld\n", lists, in_lists, p.items.size(), p.pages.size(), p.tokens.size(),
           p.merge_tokens.size(), p.sources.size(), (long long)p.n_parts);
  }
  return 0;
}
