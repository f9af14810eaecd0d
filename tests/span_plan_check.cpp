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
  std::vector<int> flat;
  for (const auto& t : p.tables) flat.insert(flat.end(), t.pages, t.pages + t.n);
  CHECK((int64_t)flat.size() == p.n_pages, "pages %zu", flat.size());
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
  for (const SpanItem& it : p.items) {
    CHECK(it.rows >= 0 && it.rows < (int)p.rows.size(), "rows");
    const SpanRows& rw = p.rows[it.rows];
    CHECK(it.kvh >= 0 && it.kvh < c.nkv && it.n_rows >= 1, "kvh %d", it.kvh);
    CHECK(it.row0 + it.n_rows <= rw.n_rows && it.n_rows <= (it.kind ? kSpanTileRows : 16), "rows of an item");
    CHECK(it.page0 % 2 == 0 && it.page0 >= 0, "page0 %d", it.page0);
    if (it.page0 >= it.page_end) CHECK(it.part >= 0, "an empty item without partials");
    if (it.kind == 0) {
      const int a = it.row0 / group, b = (it.row0 + it.n_rows - 1) / group;
      CHECK(rw.list || a == b, "a stream's rows are of one position");
      CHECK(rw.list || a == 0, "a stream's position");
    }
    std::vector<std::pair<int, int>> keys;
    for (int v = it.page0; v < it.page_end; v++) {
      const int t = v < rw.sink_pages ? v : v + it.skip;
      const int real = v < rw.sink_pages ? v : v + it.skip + rw.skip;
      CHECK(rw.pages + t >= 0 && rw.pages + t < (int)flat.size(), "table entry");
      keys.push_back({flat[rw.pages + t], rw.list ? -1 : 16 * real});
    }
    for (int i = 0; i < it.n_rows; i++) {
      const int row = it.row0 + i, tk = row / group, h = it.kvh * group + row % group;
      const int tok = rw.list ? p.tokens.at(rw.tok + tk) : rw.tok + tk;
      CHECK(tok >= 0 && tok < T, "token %d", tok);
      CHECK(rw.list || rw.pos + tk == tok_pos[tok], "position");
      if (it.part >= 0) {
        CHECK(it.part + i < p.n_parts, "partial %d of %lld", it.part + i, (long long)p.n_parts);
        CHECK(!written[it.part + i], "partial %d twice", it.part + i);
        written[it.part + i] = 1;
        at_part[it.part + i] = keys;
        part_row[it.part + i] = {tok, h};
      } else {
        got[{tok, h}].parts.push_back({-1, keys});
      }
    }
  }
  std::set<int> used;
  for (const SpanToken& tk : p.merge_tokens) {
    const SpanMerge& m = p.merges.at(tk.merge);
    int n = 0;
    for (int h = 0; h < c.nq; h++) {
      const int g = h / group;
      for (int s = 0; s < m.n_src; s++) {
        const SpanSource& src = p.sources.at(m.src + s);
        for (int k = 0; k < src.n_split; k++) {
          const int at = (tk.tok - m.tok) * group + h - g * group + src.base + g * src.kvh_stride + k * src.split_stride;
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
    const int shapes[][2] = {{4, 4}, {8, 2}, {8, 1}, {5, 5}, {20, 1}, {36, 2}, {32, 8}, {64, 8}, {150, 1}};
    const auto& s = shapes[in(0, 8)];
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
        const int pages = log_in(9);
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
