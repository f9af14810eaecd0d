// Walks the host's plans of attention over parts of the keys (span_plan.h) as the kernels do,
// for random batches: every row meets each key that it sees exactly once, reads only pages of
// its request, and finds its partials; the workspace bounds hold.  Prints what is wrong.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

#include "span_plan.h"

using namespace mx;


static int errors = 0;
#define CHECK(c, ...)                                   \
  do {                                                  \
    if (!(c) && errors++ < 20) {                        \
      printf("line %d: ", __LINE__), printf(__VA_ARGS__), printf("\n"); \
    }                                                   \
  } while (0)

struct Case {
  int nq, nkv;
  std::vector<mx_request> reqs;
  std::vector<std::vector<int>> pages;
  std::vector<mx_shared_run> runs;
  int window = 0, sinks = 0;
};

// what the items leave for (batch row, q head): page ids with first key, by partial (-1: output)
struct Got {
  std::vector<std::pair<int, std::vector<std::pair<int, int>>>> parts;
};

static void walk(const Case& c, const SpanPlan& p) {
  const int group = c.nq / c.nkv;
  const std::vector<int>& flat = p.pages;
  std::vector<int> tok_req, tok_pos;
  for (size_t r = 0; r < c.reqs.size(); r++)
    for (int i = 0; i < c.reqs[r].n_new; i++) {
      tok_req.push_back((int)r);
      tok_pos.push_back(c.reqs[r].ctx_len + i);
    }
  const int T = (int)tok_req.size();
  std::map<std::pair<int, int>, Got> got;
  std::vector<char> written(p.n_parts, 0);
  std::map<int, std::vector<std::pair<int, int>>> at_part;  // partial -> (page id, first key)
  std::map<int, std::pair<int, int>> part_row;
  for (int b = 0; b < p.blocks(); b++) {
    const SpanBlock at_b = span_block(b, (int)p.items.size(), p.nkv, p.heads);
    CHECK(at_b.item >= 0 && at_b.item < (int)p.items.size() && at_b.kvh >= 0 && at_b.kvh < p.nkv, "block %d", b);
    const SpanItem& it = p.items[at_b.item];
    CHECK(it.n_rows >= 1 && it.rest >= 0 && it.rest < group, "rows of an item");
    CHECK(it.n_rows <= (it.kind ? kSpanTileRows : kSpanStreamRows), "rows of an item");
    CHECK(it.page0 % 2 == 0 && it.page0 >= 0, "page0 %d", it.page0);
    if (it.page0 >= it.page1) CHECK(it.part >= 0, "an empty item without partials");
    std::vector<std::pair<int, int>> keys;
    for (int v = it.page0; v < it.page1; v++) {
      const int t = v < it.sink_pages ? v : v + it.skip_table;
      const int real = v < it.sink_pages ? v : v + it.skip_real;
      CHECK(it.pages + t >= 0 && it.pages + t < (int)flat.size(), "table entry");
      keys.push_back({flat[it.pages + t], it.list ? -1 : 16 * real});
    }
    for (int i = 0; i < it.n_rows; i++) {
      const int tk = (it.rest + i) / group, h = at_b.kvh * group + (it.rest + i) % group;
      const int tok = it.list ? p.tokens.at(it.tok + tk) : it.tok + tk;
      CHECK(tok >= 0 && tok < T, "token %d", tok);
      CHECK(it.list ? it.pos >= INT32_MAX - 16 : it.pos + tk == tok_pos[tok], "position");
      if (it.part >= 0) {
        const int at = it.part + at_b.kvh * it.kvh_stride + i;
        CHECK(at < p.n_parts, "partial %d of %lld", at, (long long)p.n_parts);
        CHECK(!written[at], "partial %d twice", at);
        written[at] = 1;
        at_part[at] = keys;
        part_row[at] = {tok, h};
      } else {
        got[{tok, h}].parts.push_back({-1, keys});
      }
    }
  }
  std::set<int> used;
  for (const SpanToken& tk : p.merge_tokens) {
    int n = 0;
    for (int h = 0; h < c.nq; h++) {
      const int g = h / group;
      for (int s = 0; s < tk.n_src; s++) {
        const SpanSource& src = p.sources.at(tk.src + s);
        for (int k = 0; k < src.n_split; k++) {
          const int at = src.base + g * src.kvh_stride + k * src.split_stride + tk.at * group + h - g * group;
          CHECK(at >= 0 && at < p.n_parts && written[at], "merge reads partial %d", at);
          CHECK(part_row[at] == std::make_pair(tk.tok, h), "partial %d is another row's", at);
          CHECK(used.insert(at).second, "partial %d read twice", at);
          got[{tk.tok, h}].parts.push_back({at, at_part[at]});
          n++;
        }
      }
    }
    CHECK(n <= p.most_parts * c.nq, "most_parts");
  }
  CHECK((int64_t)used.size() == p.n_parts, "%zu partials read of %lld", used.size(), (long long)p.n_parts);
  for (int t = 0; t < T; t++)
    for (int h = 0; h < c.nq; h += std::max(1, c.nq - 1)) {
      const Got& gt = got[{t, h}];
      int direct = 0;
      for (const auto& x : gt.parts) direct += x.first < 0;
      CHECK(direct == 0 || gt.parts.size() == 1, "row %d %d: output and partials", t, h);
      const int r = tok_req[t], pos = tok_pos[t];
      std::map<int, int> seen;  // page index -> times
      for (const auto& x : gt.parts)
        for (const auto& k : x.second) {
          int real = k.second / 16;
          if (k.second < 0) {  // of a run: a page whose keys all rows see
            real = -1;
            for (int i = 0; 16 * (i + 1) <= c.reqs[r].ctx_len && real < 0; i++)
              if (c.pages[r][i] == k.first) real = i;
            CHECK(real >= 0, "a run's page is not the request's");
          }
          CHECK(real >= 0 && real < (int)c.pages[r].size() && c.pages[r][real] == k.first, "row %d: page", t);
          seen[real]++;
        }
      for (int i = 0; 16 * i <= pos; i++) {
        bool some = false;
        for (int j = 16 * i; j < 16 * i + 16 && j <= pos; j++)
          some |= !c.window || j < c.sinks || j > pos - c.window;
        const int n = seen.count(i) ? seen[i] : 0;
        CHECK(n <= 1 && (!some || n == 1), "row %d (pos %d): page %d read %d times, seen %d", t, pos, i, n, some);
      }
    }
}

int main(int argc, char** argv) {
  const int n = atoi(argv[1]);
  for (int seed = 0; seed < n; seed++) {
    std::mt19937 rng(seed);
    auto in = [&](int a, int b) { return a + (int)(rng() % (unsigned)(b - a + 1)); };
    auto log_in = [&](int hi) { return in(1, 1 << in(0, hi)); };
    Case c;
    const int shapes[][2] = {{4, 4}, {8, 2}, {8, 1}, {5, 5}, {20, 1}, {36, 2}, {32, 8}, {64, 8}, {150, 1}, {20, 10}, {19, 19}};
    const auto& s = shapes[in(0, 10)];
    c.nq = s[0], c.nkv = s[1];
    const bool window = seed % 2;
    const int R = in(1, window ? 6 : 10);
    std::vector<int> start(R, 0);
    std::vector<std::vector<int>> shared(R);
    int next = 0;
    if (!window) {
      for (int k = in(0, 5); k > 0; k--) {
        const int first = in(0, R - 1), num = in(1, R - first);
        bool same = true;
        for (int r = first; r < first + num; r++) same &= shared[r].size() == shared[first].size();
        if (!same) continue;
        const int pages = log_in(in(0, 3) ? 8 : 12);
        for (int i = 0; i < pages; i++, next++)
          for (int r = first; r < first + num; r++) shared[r].push_back(next);
        c.runs.push_back({first, num, pages});
      }
    }
    for (int r = 0; r < R; r++) {
      const bool decode = in(0, 1);
      const int n_new = decode ? 1 : log_in(10);
      const int ctx = 16 * (int)shared[r].size() + in(0, 2) * (log_in(window ? 13 : 10) - 1) + (decode && shared[r].empty());
      std::vector<int> pg = shared[r];
      while ((int)pg.size() * 16 < ctx + n_new) pg.push_back(next++);
      c.pages.push_back(pg);
      c.reqs.push_back({decode ? MX_DECODE : MX_PREFILL, n_new, ctx, (int)pg.size(), nullptr});
    }
    for (int r = 0; r < R; r++) c.reqs[r].pages = c.pages[r].data();
    const mx_batch b{R, c.reqs.data()};
    const mx_attn_shape shape{c.nq, c.nkv, 64, 16, next, 0.f};
    SpanPlan p;
    if (window) {
      c.window = log_in(12), c.sinks = in(0, 1) * log_in(9);
      if (in(0, 9) == 0) c.window = INT32_MAX;
      plan_window(&b, &shape, c.window, c.sinks, p);
    } else {
      if (in(0, 3)) p.min_shared_bytes = 0;
      plan_shared(&b, &shape, (int)c.runs.size(), c.runs.data(), p);
    }
    const int before = errors;
    walk(c, p);
    if (errors > before) printf("seed %d: %d q heads, %d KV heads, window %d, sinks %d\n", seed, c.nq, c.nkv, c.window, c.sinks);
    if (errors > 20) break;
  }
  printf("%d errors\n", errors);
  return errors != 0;
}
