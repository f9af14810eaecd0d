// attention_span.hip -- paged attention that does not scan a request's whole cache by
// itself: with a sliding window and sinks, and over runs of pages that requests share.
//
// A token at position p sees the keys j <= p with j < sinks or j > p - window.  The host
// lists, for rows that share their keys, the pages that some of them sees; an item takes a
// range of that list for rows of one KV head.  The q heads of a KV head's group are rows of
// one item, so keys are read once for the group, and a tile's rows, 128 / group consecutive
// tokens, see nearly the same keys.  Everything else is the arithmetic of the bf16
// attention: S^T = K Q^T and O^T += V^T P^T with the 16x16x32 matrix instruction, a row's
// softmax in the four lanes that hold it.
//
// Rows with several items (split keys; shared and own keys) leave unnormalised outputs,
// maxima and sums in fp32, which a second launch joins in a fixed order.
//
// Masked scores are -inf and a row's running maximum starts at the lowest finite number, so
// that a row without a key in an item's chunk, or in the whole item, adds exactly 0.
#include <type_traits>

#include "attention_bf16.h"
#include "attention_span.h"

namespace mx {

namespace {

constexpr float kLowest = -3.402823466e38f, kInf = __builtin_inff();
__device__ __forceinline__ RowState span_row_start() { return RowState{kLowest, -kInf, 0.f}; }

// Where an item's pages lie, and what a position sees of them.
struct Span {
  int sink_pages, skip_table, skip_real, page_end, window, sinks;
  __device__ __forceinline__ Span(const SpanParams& p, const SpanItem& it, const SpanRows& rw)
      : sink_pages(rw.sink_pages), skip_table(it.skip), skip_real(it.skip + rw.skip),
        page_end(it.page_end), window(p.window), sinks(p.sinks) {}
  __device__ __forceinline__ int entry(int v) const { return v < sink_pages ? v : v + skip_table; }
  __device__ __forceinline__ int first_key(int v) const {  // of page v, as a position
    return 16 * (v < sink_pages ? v : v + skip_real);
  }
  __device__ __forceinline__ bool sees(int pos, int key) const {
    return key <= pos && (key < sinks || key > pos - window);
  }
  // pages v and v + 1 are in the item, and all their keys seen from pos0 .. pos1
  __device__ __forceinline__ bool all_seen(int v, int pos0, int pos1) const {
    if (v + 1 >= page_end) return false;
    const int first = first_key(v), last = first_key(v + 1) + 15;
    return last <= pos0 && (first > pos1 - window || last < sinks);
  }
  // some key of the pages may be seen from pos0 .. pos1
  __device__ __forceinline__ bool some_seen(int v, int pos0, int pos1) const {
    const int first = first_key(v), last = first_key(min(v + 1, page_end - 1)) + 15;
    return first <= pos1 && (first < sinks || last > pos0 - window);
  }
};

// Which of the lane group's eight keys (all of one page) the row at pos sees, as bits.
__device__ __forceinline__ unsigned seen_keys(const Span& s, int v0, int pos, int g4) {
  const int v = v0 + (g4 >> 1);
  if (v >= s.page_end) return 0;
  const int j0 = s.first_key(v) + 8 * (g4 & 1);
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) m |= s.sees(pos, j0 + e) ? 1u << e : 0u;
  return m;
}
__device__ __forceinline__ float mask_scores(const f32x4 (&s)[2], float (&sv)[2][4], unsigned seen) {
  float mx = -kInf;
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      sv[b][i] = seen >> (4 * b + i) & 1 ? s[b][i] : -kInf;
      mx = fmaxf(mx, sv[b][i]);
    }
  return mx;
}
__device__ __forceinline__ float take_scores(const f32x4 (&s)[2], float (&sv)[2][4]) {
  float mx = -kInf;
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      sv[b][i] = s[b][i];
      mx = fmaxf(mx, sv[b][i]);
    }
  return mx;
}
// The keys' bits as a mask on their values (two keys a word).
__device__ __forceinline__ void value_mask(unsigned seen, uint32_t (&keep)[4]) {
#pragma unroll
  for (int h = 0; h < 4; h++)
    keep[h] = (seen >> (2 * h) & 1 ? 0xFFFFu : 0u) | (seen >> (2 * h + 1) & 1 ? 0xFFFF0000u : 0u);
}

// Values that are no numbers, where only some rows see their keys: a probability of 0 would
// not keep them out of the other rows' sums, so they are taken out of the products and come
// back through products of their own, of their places with the keys that a row sees (ones).
// Needed in chunks on the edge of what a tile's rows see; a search over their values there
// (two instructions a word) finds when.
__device__ __forceinline__ bool some_not_finite(const u32x4& v) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) t |= (v[i] & 0x7F807F80u) + 0x00800080u;
  return (t & 0x80008000u) != 0;
}
__device__ __forceinline__ bf16x8 seen_ones(unsigned seen) {
  uint32_t keep[4];
  value_mask(seen, keep);
  return as_bf16x8(u32x4{keep[0] & 0x3F803F80u, keep[1] & 0x3F803F80u, keep[2] & 0x3F803F80u,
                         keep[3] & 0x3F803F80u});
}
__device__ __forceinline__ void put_not_finite(const u32x4& v, unsigned seen, f32x4& o) {
  u32x4 nan, up, down;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    nan[i] = up[i] = down[i] = 0;
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const uint32_t x = v[i] >> h & 0xFFFFu;
      nan[i] |= (x & 0x7FFFu) > 0x7F80u ? 0x3F80u << h : 0u;
      up[i] |= x == 0x7F80u ? 0x3F80u << h : 0u;
      down[i] |= x == 0xFF80u ? 0x3F80u << h : 0u;
    }
  }
  const bf16x8 ones = seen_ones(seen);
  const f32x4 zero = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4 n = mfma16(as_bf16x8(nan), ones, zero), u = mfma16(as_bf16x8(up), ones, zero),
              d = mfma16(as_bf16x8(down), ones, zero);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (n[i] > 0.f) o[i] = __builtin_nanf("");
    if (u[i] > 0.f) o[i] += kInf;
    if (d[i] > 0.f) o[i] -= kInf;
  }
}
__device__ __forceinline__ void drop_not_finite(u32x4& v) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if ((v[i] & 0x7F80u) == 0x7F80u) v[i] &= 0xFFFF0000u;
    if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] &= 0xFFFFu;
  }
}

// A row's place in the batch.
struct RowAt {
  int64_t tok;
  int head, pos;
};
__device__ __forceinline__ RowAt row_at(const SpanParams& p, const SpanRows& rw, int kvh, int row) {
  const int t = row / p.a.group, h = kvh * p.a.group + row - t * p.a.group;
  if (rw.list) return RowAt{p.tokens[rw.tok + t], h, rw.pos};
  return RowAt{rw.tok + t, h, rw.pos + t};
}

static_assert(kSpanTileRows == 4 * 32, "four waves of two 16-row blocks");
// Tile: 128 rows, 32 of each wave in two blocks of 16, over 32-key chunks that the four
// waves share through LDS, as the bf16 attention's prefill tiles (prefill_item there tells
// how the copies run three chunks ahead).  Chunks that all rows of the tile see whole, from
// first_whole to end_whole, take no masks; those before (the window's low edge, sinks) and
// behind (the diagonal, the end) do, and a wave leaves out those that none of its rows sees.
template <int HD>
__device__ __forceinline__ void tile_item(const SpanParams& p, const SpanItem& it, const SpanRows& rw,
                                          char* smem) {
  using SC = SharedChunk<HD>;
  constexpr int KB = SC::KBYTES, CB = SC::BYTES, NLD = SC::NLD, ND = HD / 32;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // row of this lane within each block
  const int g4 = lane >> 4;   // lane group
  const int kvh = it.kvh;
  const Span span(p, it, rw);
  const int end_row = it.row0 + it.n_rows;
  const int row0 = it.row0 + 32 * wave;
  const int first_page = it.page0, page_end = it.page_end;
  const int n_chunks = (page_end - first_page + 1) / 2;

  bf16x8 qf[ND], qf2[ND];
  int pos, pos2;
  {
    auto load = [&](int row, bf16x8 (&f)[ND], int& at) {
      const RowAt r = row_at(p, rw, kvh, min(row, end_row - 1));
      const uint16_t* qp = p.a.q + r.tok * p.a.q_tok_stride + (int64_t)r.head * HD + 8 * g4;
#pragma unroll
      for (int ds = 0; ds < ND; ds++) f[ds] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ds * 32));
      at = r.pos;
    };
    load(row0 + col, qf, pos);
    load(row0 + 16 + col, qf2, pos2);
  }
  RowState r1 = span_row_start(), r2 = span_row_start();
  const float scale = p.a.scale_log2, inv_scale = 1.f / scale;
  f32x4 o[HD / 16], o2[HD / 16];
#pragma unroll
  for (int db = 0; db < HD / 16; db++) o[db] = o2[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  // positions of the tile's rows and of the wave's
  auto pos_of = [&](int row) {
    return rw.list ? rw.pos : rw.pos + min(row, end_row - 1) / p.a.group;
  };
  const int tile_pos0 = pos_of(it.row0), tile_pos1 = pos_of(end_row - 1);
  const int wave_pos0 = pos_of(row0), wave_pos1 = pos_of(row0 + 31);

  // the chunks that need no mask: first_whole .. end_whole - 1
  int first_whole = 0, end_whole;
  {
    const int low = tile_pos1 - span.window + 1;  // the first key that the last row's window holds
    if (low > span.sinks)
      first_whole = (max(span.sink_pages, (low + 15) / 16 - span.skip_real) - first_page + 1) / 2;
    const int last = tile_pos0 >= 15 ? (tile_pos0 - 15) / 16 - span.skip_real : -1;  // page all rows see
    end_whole = (min(page_end - 1, last) - first_page + 1) / 2;
    first_whole = min(max(first_whole, 0), n_chunks);
    end_whole = max(end_whole, first_whole);
  }

  // page ids through the constant address space: uniform reads of a table nothing writes
  // during the launch, so they are scalar loads
  const __attribute__((address_space(4))) int32_t* ptab =
      (const __attribute__((address_space(4))) int32_t*)(p.a.pages + rw.pages);
  unsigned off[NLD];  // this lane's shares of the wave's copies, bytes from the page's start
#pragma unroll
  for (int i = 0; i < NLD; i++) {
    const int kb = NLD * wave + i;
    if (wave < 2) {
      constexpr int lanes_per_row = HD / 8;
      const int j = kb * (64 / lanes_per_row) + lane / lanes_per_row;
      const int lc = (lane % lanes_per_row) ^ ksw<HD>(j);
      off[i] = 2 * ((lc >> 2) * 512 + (j & 15) * 32 + (lc & 3) * 8);
    } else {
      off[i] = (unsigned)(((kb - KB / 1024) * 1024 + lane * 16) % (HD * 32));
    }
  }
  const char* pool = (const char*)(wave < 2 ? p.a.k_pool : p.a.v_pool) + (int64_t)kvh * (32 * HD);
  const int64_t page_bytes = (int64_t)p.a.nkv * (32 * HD);
  const unsigned lds0 = (unsigned)(size_t)(MX_LDS char*)smem;
  const unsigned dst0 = lds0 + (unsigned)(NLD * wave * 1024);
  auto copy = [&](int c, int page) {
    const char* base = pool + page * page_bytes;
    const unsigned dst = dst0 + (unsigned)((c & 3) * CB);
#pragma unroll
    for (int i = 0; i < NLD; i++) dma16_at(base, off[i], dst + i * 1024);
  };
  // the page this wave copies of chunk c (past the item's last page: that page)
  auto page_of = [&](int c) {
    return ptab[span.entry(min(first_page + 2 * c + (wave & 1), page_end - 1))];
  };
  const int key0 = 16 * (col >> 3) + 8 * ((col >> 2) & 1) + (col & 3);
  unsigned kaddr[ND];
#pragma unroll
  for (int ds = 0; ds < ND; ds++)
    kaddr[ds] = lds0 + (unsigned)(key0 * (HD * 2) + (((4 * ds + g4) ^ ksw<HD>(key0)) << 4));
  const unsigned vaddr = lds0 + (unsigned)(KB + (g4 >> 1) * (HD * 32) + col * 32 + ((g4 & 1) << 4));

  float sv1[2][4], sv2[2][4], mx1 = -kInf, mx2 = -kInf;
  auto scores = [&](auto mask, auto slot, int c) -> bool {
    constexpr bool MASK = decltype(mask)::value;
    u32x4 k0[ND], k1[ND];
    if constexpr (decltype(slot)::value >= 0) {
      constexpr int OFF = decltype(slot)::value * CB;
#pragma unroll
      for (int ds = 0; ds < ND; ds++) k0[ds] = lds_read16_at<OFF>(kaddr[ds]);
#pragma unroll
      for (int ds = 0; ds < ND; ds++) k1[ds] = lds_read16_at<OFF + 4 * HD * 2>(kaddr[ds]);
    } else {
      const unsigned sb = (unsigned)((c & 3) * CB);
#pragma unroll
      for (int ds = 0; ds < ND; ds++) k0[ds] = lds_read16(sb + kaddr[ds]);
#pragma unroll
      for (int ds = 0; ds < ND; ds++) k1[ds] = lds_read16_at<4 * HD * 2>(sb + kaddr[ds]);
    }
    f32x4 s1[2], s2[2];
    lgkm_wait<ND>();
    pin(k0);
    s1[0] = score_block<HD>(k0, qf);
    s2[0] = score_block<HD>(k0, qf2);
    __builtin_amdgcn_sched_barrier(0);  // these products go before the second wait
    lgkm_wait<0>();
    pin(k1);
    s1[1] = score_block<HD>(k1, qf);
    s2[1] = score_block<HD>(k1, qf2);
    if constexpr (MASK) {
      mx1 = mask_scores(s1, sv1, seen_keys(span, first_page + 2 * c, pos, g4));
      mx2 = mask_scores(s2, sv2, seen_keys(span, first_page + 2 * c, pos2, g4));
    } else {
      mx1 = take_scores(s1, sv1);
      mx2 = take_scores(s2, sv2);
    }
    return __any(mx1 > r1.thr || mx2 > r2.thr) != 0;
  };
  auto values = [&](auto mask, auto slot, int c, bf16x8 pb1, bf16x8 pb2) {
    constexpr bool MASK = decltype(mask)::value;
    constexpr int OFF = decltype(slot)::value >= 0 ? decltype(slot)::value * CB : 0;
    const unsigned va = decltype(slot)::value >= 0 ? vaddr : vaddr + (unsigned)((c & 3) * CB);
    u32x4 v0[ND], v1[ND];
    lds_read_run<0, ND, OFF, 512>(va, v0);
    lds_read_run<0, ND, OFF + ND * 512, 512>(va, v1);
    const uint32_t none[4] = {};
    auto part = [&](auto first, u32x4 (&v)[ND]) {
      constexpr int DB0 = decltype(first)::value;
      if constexpr (MASK) {
        bool some = false;
#pragma unroll
        for (int e = 0; e < ND; e++) some |= some_not_finite(v[e]);
        if (__any(some)) {
          const unsigned n1 = seen_keys(span, first_page + 2 * c, pos, g4);
          const unsigned n2 = seen_keys(span, first_page + 2 * c, pos2, g4);
#pragma unroll
          for (int e = 0; e < ND; e++) {
            put_not_finite(v[e], n1, o[DB0 + e]);
            put_not_finite(v[e], n2, o2[DB0 + e]);
            drop_not_finite(v[e]);
          }
        }
      }
      values_part<HD, DB0, ND, false>(v, o, pb1, none);
      values_part<HD, DB0, ND, false>(v, o2, pb2, none);
    };
    // (no branch may come between a read and its wait)
    lgkm_wait<MASK ? 0 : ND>();
    pin(v0);
    if constexpr (MASK) pin(v1);
    part(std::integral_constant<int, 0>{}, v0);
    if constexpr (!MASK) {
      __builtin_amdgcn_sched_barrier(0);  // these products go before the second wait
      lgkm_wait<0>();
      pin(v1);
    }
    part(std::integral_constant<int, ND>{}, v1);
  };
  auto raise_rows = [&]() {
    raise_max(r1, mx1, scale, inv_scale, o);
    raise_max(r2, mx2, scale, inv_scale, o2);
  };
  using Masked = std::integral_constant<bool, true>;
  using Unmasked = std::integral_constant<bool, false>;
  using AnySlot = std::integral_constant<int, -1>;

  int ua, fa = 0;  // page of the chunk the next copy is for, and of the one after
  {
    const int a0 = page_of(0), a1 = page_of(1), a2 = page_of(2);
    copy(0, a0);
    copy(1, a1);
    ua = page_of(3);
    copy(2, a2);
  }
  // top of iteration kt: this wave's copies of chunk kt + 1 have landed, then everyone's,
  // and every read of chunk kt - 1 is done; chunk kt + 3 goes out
  auto top = [&](int kt, int& use, int& fill) {
    vm_wait<NLD>();
    wg_barrier();
    fill = page_of(kt + 4);
    copy(kt + 3, use);
  };
  auto run = [&](int kt0, int kt1, auto body) {  // iterations kt0 .. kt1 - 1
    for (int kt = kt0; kt < kt1; kt += 2) {
      top(kt, ua, fa);
      body(kt);
      if (kt + 1 >= kt1) {  // an odd count: the next iteration uses fa
        const int t = ua;
        ua = fa;
        fa = t;
        break;
      }
      top(kt + 1, fa, ua);
      body(kt + 1);
    }
  };

  if (row0 >= end_row) {
    // no rows here: this wave only copies its quarter of every chunk
    vm_wait<2 * NLD>();
    wg_barrier();
    run(0, n_chunks, [](int) {});
    vm_wait<0>();  // no copy may land in LDS after the workgroup has ended
    return;
  }
  auto takes = [&](int c) {
    return c < n_chunks && span.some_seen(first_page + 2 * c, wave_pos0, wave_pos1);
  };
  vm_wait<2 * NLD>();  // chunk 0 has landed; chunks 1 and 2 may be in flight
  wg_barrier();
  if (takes(0) && scores(Masked{}, AnySlot{}, 0)) raise_rows();

  // Iteration kt holds the scores of chunk kt (of the previous iteration), takes its
  // softmax and values, and the scores of chunk kt + 1.
  auto edge = [&](int kt) {
    if (takes(kt)) {
      const bf16x8 pb1 = probs(sv1, r1, scale);
      const bf16x8 pb2 = probs(sv2, r2, scale);
      values(Masked{}, AnySlot{}, kt, pb1, pb2);
    }
    if (takes(kt + 1) && scores(Masked{}, AnySlot{}, kt + 1)) raise_rows();
  };
  // the scores of chunk kt + 1 and the softmax of chunk kt in one basic block, then the
  // values of chunk kt; no masks
  auto step = [&](auto slot, int kt) {  // slot: kt % 4 or -1
    constexpr int S = decltype(slot)::value, S1 = S < 0 ? -1 : (S + 1) % 4;
    const bf16x8 pb1 = probs(sv1, r1, scale);
    const bf16x8 pb2 = probs(sv2, r2, scale);
    const bool raise = scores(Unmasked{}, std::integral_constant<int, S1>{}, kt + 1);
    values(Unmasked{}, slot, kt, pb1, pb2);
    if (raise) raise_rows();
  };
  // the whole chunks' iterations: both kt and kt + 1 are whole, from a multiple of four on
  // four at a time, whose ring slots are constants in the fragment reads
  const int main0 = first_whole, main1 = max(end_whole - 1, main0);
  const int four0 = min((main0 + 3) & ~3, main1), four1 = four0 + ((main1 - four0) & ~3);
  run(0, main0, edge);
  run(main0, four0, [&](int kt) { step(AnySlot{}, kt); });
  for (int kt = four0; kt < four1; kt += 4) {
    top(kt, ua, fa);
    step(std::integral_constant<int, 0>{}, kt);
    top(kt + 1, fa, ua);
    step(std::integral_constant<int, 1>{}, kt + 1);
    top(kt + 2, ua, fa);
    step(std::integral_constant<int, 2>{}, kt + 2);
    top(kt + 3, fa, ua);
    step(std::integral_constant<int, 3>{}, kt + 3);
  }
  run(four1, main1, [&](int kt) { step(AnySlot{}, kt); });
  run(main1, n_chunks, edge);
  vm_wait<0>();  // no copy may land in LDS after the workgroup has ended

  // the rows' sums over their four lane groups (every lane takes part)
  const float l1 = lane_groups_sum(r1.l), l2 = lane_groups_sum(r2.l);
  const int64_t step32 = p.a.out_tiled ? 512 : 32;
  auto store = [&](int row, float l, const RowState& st, const f32x4 (&acc)[HD / 16]) {
    if (row >= end_row) return;
    if (it.part >= 0) {
      const int64_t part = (int64_t)it.part + row - it.row0;
#pragma unroll
      for (int db = 0; db < HD / 16; db++)
        *reinterpret_cast<f32x4*>(p.a.part_o + part * HD + 16 * db + 4 * g4) = acc[db];
      if (g4 == 0) *reinterpret_cast<float2*>(p.a.part_ml + 2 * part) = float2{st.m, l};
      return;
    }
    const RowAt r = row_at(p, rw, kvh, row);
    const float inv = 1.f / l;
    uint16_t* op = out_ptr(p.a, r.tok, r.head * HD + 4 * g4);
#pragma unroll
    for (int db = 0; db < HD / 16; db++) {
      u32x2 w;
      w[0] = pack_bf16x2(acc[db][0] * inv, acc[db][1] * inv);
      w[1] = pack_bf16x2(acc[db][2] * inv, acc[db][3] * inv);
      *reinterpret_cast<u32x2*>(op + (db >> 1) * step32 + (db & 1) * 16) = w;
    }
  };
  store(row0 + col, l1, r1, o);
  store(row0 + 16 + col, l2, r2, o2);
}

// Stream: up to 16 rows of one position (a decode's q heads; or rows that see a whole run);
// the four waves stride over the item's 32-key chunks, keys and values straight to
// registers, and combine through LDS.  Keys that the rows do not see are taken out by
// select, scores and values, so what their slots hold stays out.
template <int HD, bool NT>
__device__ __forceinline__ void stream_item(const SpanParams& p, const SpanItem& it, const SpanRows& rw,
                                            char* smem) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int col = lane & 15;  // row of this lane
  const int g4 = lane >> 4;   // lane group
  const int kvh = it.kvh, page_end = it.page_end;
  const Span span(p, it, rw);
  const RowAt at = row_at(p, rw, kvh, it.row0 + min(col, it.n_rows - 1));
  const int pos = rw.list ? rw.pos : rw.pos + it.row0 / p.a.group;  // of every row
  RowState r = span_row_start();
  const float scale = p.a.scale_log2, inv_scale = 1.f / scale;
  f32x4 o[HD / 16];
#pragma unroll
  for (int db = 0; db < HD / 16; db++) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 qf[HD / 32];
  {
    const uint16_t* qp = p.a.q + at.tok * p.a.q_tok_stride + (int64_t)at.head * HD + 8 * g4;
#pragma unroll
    for (int ds = 0; ds < HD / 32; ds++) qf[ds] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ds * 32));
  }
  const int32_t* ptab = p.a.pages + rw.pages;
  auto pid = [&](int v) { return ptab[span.entry(min(v, page_end - 1))]; };
  auto proc = [&](Chunk<HD>& c, int v) {
    const f32x4 s[2] = {score_block<HD>(c.k[0], qf), score_block<HD>(c.k[1], qf)};
    float sv[2][4];
    float mx = take_scores(s, sv);
    if (!span.all_seen(v, pos, pos)) {
      const unsigned seen = seen_keys(span, v, pos, g4);
      mx = mask_scores(s, sv, seen);
      uint32_t keep[4];
      value_mask(seen, keep);
#pragma unroll
      for (int db = 0; db < HD / 16; db++)
#pragma unroll
        for (int h = 0; h < 4; h++) c.v[db][h] &= keep[h];
    }
    if (__any(mx > r.thr)) raise_max(r, mx, scale, inv_scale, o);
    const bf16x8 pb = probs(sv, r, scale);
    const uint32_t none[4] = {};
    values_part<HD, 0, HD / 16, false>(c.v, o, pb, none);
  };
  // two chunk buffers in turn, a chunk's loads issued only where it exists (decode_item of
  // the bf16 attention tells why)
  constexpr int STEP = 8;
  Chunk<HD> ca, cb;
  int v = it.page0 + 2 * wave;
  if (v < page_end) {
    int n0 = pid(v + STEP), n1 = pid(v + STEP + 1);
    load_chunk<HD, NT>(ca, p.a, kvh, pid(v), pid(v + 1), 0, col, g4);
    while (true) {
      int vn = v + STEP;
      if (vn >= page_end) {
        proc(ca, v);
        break;
      }
      int m0 = pid(vn + STEP), m1 = pid(vn + STEP + 1);
      load_chunk<HD, NT>(cb, p.a, kvh, n0, n1, 0, col, g4);
      proc(ca, v);
      v = vn;
      n0 = m0;
      n1 = m1;
      vn = v + STEP;
      if (vn >= page_end) {
        proc(cb, v);
        break;
      }
      m0 = pid(vn + STEP);
      m1 = pid(vn + STEP + 1);
      load_chunk<HD, NT>(ca, p.a, kvh, n0, n1, 0, col, g4);
      proc(cb, v);
      v = vn;
      n0 = m0;
      n1 = m1;
    }
  }

  float(*s_o)[16][HD + 4] = reinterpret_cast<float(*)[16][HD + 4]>(smem);
  float(*s_m)[16] = reinterpret_cast<float(*)[16]>(smem + 4 * 16 * (HD + 4) * 4);
  float(*s_l)[16] = reinterpret_cast<float(*)[16]>(smem + 4 * 16 * (HD + 4) * 4 + 4 * 16 * 4);
#pragma unroll
  for (int db = 0; db < HD / 16; db++)
    *reinterpret_cast<f32x4*>(&s_o[wave][col][db * 16 + 4 * g4]) = o[db];
  const float l = lane_groups_sum(r.l);
  if (g4 == 0) {
    s_m[wave][col] = r.m;
    s_l[wave][col] = l;
  }
  __syncthreads();
  const int row = threadIdx.x >> 4;  // 16 rows
  const int dseg = (threadIdx.x & 15) * (HD / 16);
  if (row >= it.n_rows) return;
  float M = kLowest;
#pragma unroll
  for (int w = 0; w < 4; w++) M = fmaxf(M, s_m[w][row]);
  float wt[4], L = 0.f;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    wt[w] = exp2f(s_m[w][row] - M);
    L += s_l[w][row] * wt[w];
  }
  float acc[HD / 16];
#pragma unroll
  for (int e = 0; e < HD / 16; e++) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) a += s_o[w][row][dseg + e] * wt[w];
    acc[e] = a;
  }
  if (it.part < 0) {
    const RowAt to = row_at(p, rw, kvh, it.row0 + row);
    const float inv = 1.f / L;
    uint16_t* op = out_ptr(p.a, to.tok, to.head * HD + dseg);  // HD / 16 dims within a 32-column block
#pragma unroll
    for (int e = 0; e < HD / 16; e += 2)
      *reinterpret_cast<uint32_t*>(op + e) = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
  } else {
    const int64_t part = (int64_t)it.part + row;
    float* po = p.a.part_o + part * HD + dseg;
#pragma unroll
    for (int e = 0; e < HD / 16; e += 4)
      *reinterpret_cast<f32x4*>(po + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
    if ((threadIdx.x & 15) == 0) *reinterpret_cast<float2*>(p.a.part_ml + 2 * part) = float2{M, L};
  }
}

// An item without pages: partials that count as nothing.
template <int HD>
__device__ __forceinline__ void empty_item(const SpanParams& p, const SpanItem& it) {
  for (int i = threadIdx.x; i < it.n_rows * (HD / 4); i += 256)
    *reinterpret_cast<f32x4*>(p.a.part_o + (int64_t)it.part * HD + 4 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
  if ((int)threadIdx.x < it.n_rows)
    *reinterpret_cast<float2*>(p.a.part_ml + 2 * ((int64_t)it.part + threadIdx.x)) = float2{kLowest, 0.f};
}

template <int HD>
constexpr int combine_bytes() {
  return (4 * 16 * (HD + 4) + 2 * 4 * 16) * 4;
}
template <int HD, bool TILES>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void span_attn_kernel(SpanParams p) {
  __shared__ __attribute__((aligned(16))) char smem[TILES ? smem_bytes<HD>() : combine_bytes<HD>()];
  const SpanItem it = p.items[blockIdx.x];
  const SpanRows rw = p.rows[it.rows];
  if (it.page0 >= it.page_end) {
    empty_item<HD>(p, it);
    return;
  }
  if constexpr (TILES) {
    if (it.kind == 1) tile_item<HD>(p, it, rw, smem);
    else stream_item<HD, false>(p, it, rw, smem);
  } else {
    stream_item<HD, true>(p, it, rw, smem);
  }
}

// The merge: HD / 4 threads hold a row; a workgroup takes 8 (HD = 128) or 16 q heads of a
// token, or (WIDE) one q head, whose partials its groups of threads read side by side.
template <int HD, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void span_merge_kernel(SpanParams p, const SpanToken* tokens,
                                                                   const SpanMerge* merges,
                                                                   const SpanSource* sources) {
  constexpr int TPR = HD / 4, G = kMergeThreads / TPR;
  const SpanToken tk = tokens[blockIdx.x];
  const SpanMerge mg = merges[tk.merge];
  const int g = threadIdx.x / TPR, d = 4 * (threadIdx.x % TPR);
  const int h = WIDE ? (int)blockIdx.y : (int)blockIdx.y * G + g;
  if (!WIDE && h >= p.a.nq) return;
  const int kvh = h / p.a.group;
  const int64_t in = (int64_t)(tk.tok - mg.tok) * p.a.group + h - kvh * p.a.group;
  float m = kLowest, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  int first = WIDE ? g : 0;  // of the next source's splits
  for (int s = 0; s < mg.n_src; s++) {
    const SpanSource src = sources[mg.src + s];
    const int64_t base = in + src.base + (int64_t)kvh * src.kvh_stride;
    int k = first;
#pragma unroll 4
    for (; k < src.n_split; k += WIDE ? G : 1) {
      const int64_t at = base + (int64_t)k * src.split_stride;
      const float2 ml = *reinterpret_cast<const float2*>(p.a.part_ml + 2 * at);
      const f32x4 o = *reinterpret_cast<const f32x4*>(p.a.part_o + at * HD + d);
      const float mn = fmaxf(m, ml.x);
      const float a = exp2f(m - mn), w = exp2f(ml.x - mn);
      acc = acc * a + o * w;
      l = l * a + ml.y * w;
      m = mn;
    }
    if (WIDE) first = k - src.n_split;
  }
  if constexpr (WIDE) {
    __shared__ float s_acc[G][HD], s_m[G], s_l[G];
    *reinterpret_cast<f32x4*>(&s_acc[g][d]) = acc;
    if (d == 0) {
      s_m[g] = m;
      s_l[g] = l;
    }
    __syncthreads();
    if (threadIdx.x >= HD / 2) return;
    float M = kLowest;
#pragma unroll
    for (int k = 0; k < G; k++) M = fmaxf(M, s_m[k]);
    float L = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int k = 0; k < G; k++) {
      const float w = exp2f(s_m[k] - M);
      L += s_l[k] * w;
      a0 += s_acc[k][2 * threadIdx.x] * w;
      a1 += s_acc[k][2 * threadIdx.x + 1] * w;
    }
    *reinterpret_cast<uint32_t*>(out_ptr(p.a, tk.tok, h * HD + 2 * threadIdx.x)) =
        pack_bf16x2(a0 / L, a1 / L);
  } else {
    u32x2 w;
    w[0] = pack_bf16x2(acc[0] / l, acc[1] / l);
    w[1] = pack_bf16x2(acc[2] / l, acc[3] / l);
    *reinterpret_cast<u32x2*>(out_ptr(p.a, tk.tok, h * HD + d)) = w;
  }
}

template <int HD>
hipError_t launch(const SpanParams& p, int n_items, bool tiles, const SpanToken* merge, int n_merge,
                  bool wide, const SpanMerge* merges, const SpanSource* sources, hipStream_t stream) {
  if (n_items > 0) {
    if (tiles) span_attn_kernel<HD, true><<<n_items, 256, 0, stream>>>(p);
    else span_attn_kernel<HD, false><<<n_items, 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (n_merge == 0) return hipSuccess;
  constexpr int G = kMergeThreads / (HD / 4);
  if (wide) span_merge_kernel<HD, true><<<dim3(n_merge, p.a.nq), kMergeThreads, 0, stream>>>(p, merge, merges, sources);
  else span_merge_kernel<HD, false><<<dim3(n_merge, (p.a.nq + G - 1) / G), kMergeThreads, 0, stream>>>(p, merge, merges, sources);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_span_attn(const SpanParams& p, int n_items, bool tiles, const SpanToken* merge,
                            int n_merge, bool wide, const SpanMerge* merges,
                            const SpanSource* sources, int head_dim, hipStream_t stream) {
  const auto call = head_dim == 128 ? launch<128> : launch<64>;
  return call(p, n_items, tiles, merge, n_merge, wide, merges, sources, stream);
}

}  // namespace mx
