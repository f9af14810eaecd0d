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
// maxima and sums in fp32, which a second launch joins in a fixed order.  (Joined by the last
// of them to end instead, behind fences or with partials written through to memory, a call
// takes 8 to 250 us more; the launch takes 4 to 6.)
//
// Probabilities are rounded to bf16 for the value product, by up to 2^-8 of each; the row sums
// are those of the rounded ones, so that the errors of numerator and denominator go together.
// Scores, maxima, sums and outputs stay in fp32 up to the one rounding of the result.
//
// Masked scores are -inf and a row's running maximum starts at the lowest finite number, so
// that a row without a key in an item's chunk, or in the whole item, adds exactly 0.
#include <type_traits>

#include "attention_bf16.h"
#include "attention_span.h"

namespace mx {

namespace {

constexpr int kWaves = 4;  // of a workgroup
constexpr float kLowest = -3.402823466e38f, kInf = __builtin_inff();
__device__ __forceinline__ RowState span_row_start() { return RowState{kLowest, -kInf, 0.f}; }

// Where an item's pages lie, and what a position sees of them.
struct Span {
  int sink_pages, skip_table, skip_real, page_end, window, sinks;
  __device__ __forceinline__ Span(const SpanParams& p, const SpanItem& it)
      : sink_pages(it.sink_pages), skip_table(it.skip_table), skip_real(it.skip_real),
        page_end(it.page1), window(p.window), sinks(p.sinks) {}
  __device__ __forceinline__ int entry(int v) const { return v < sink_pages ? v : v + skip_table; }
  __device__ __forceinline__ int first_key(int v) const {  // of page v, as a position
    return 16 * (v < sink_pages ? v : v + skip_real);
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

// Which of the lane group's eight keys of pages v0 and v0 + 1 (all of one page) are seen from
// some position of pos0 .. pos1, as bits.
__device__ __forceinline__ unsigned seen_keys(const Span& s, int v0, int pos0, int pos1, int g4) {
  const int v = v0 + (g4 >> 1);
  const int j0 = s.first_key(v) + 8 * (g4 & 1);
  auto below = [](int n) { return (1u << min(max(n, 0), 8)) - 1; };  // keys j0 .. j0 + n - 1
  // (the max first: a window of 2^31 - 1 and keys behind pos0 would pass the 32 bits)
  const int hidden = max(pos0 - s.window + 1, j0) - j0;
  const unsigned m = below(pos1 - j0 + 1) & (~below(hidden) | below(s.sinks - j0));
  return v < s.page_end ? m : 0;
}
__device__ __forceinline__ unsigned seen_keys(const Span& s, int v0, int pos, int g4) {
  return seen_keys(s, v0, pos, pos, g4);
}
// The scores of these keys, -inf where the row does not see one (its bit as a word of its
// own, and a select by it), and their max.
__device__ __forceinline__ float mask_scores(const f32x4 (&s)[2], float (&sv)[2][4], unsigned seen) {
  float mx = -kInf;
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t on = (uint32_t)((int)(seen << (31 - 4 * b - i)) >> 31);
      sv[b][i] = __uint_as_float((on & __float_as_uint(s[b][i])) | (~on & 0xFF800000u));
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
// back at the item's end through products of their own, of their places with the keys that a
// row sees (ones).  Needed in chunks on the edge of what a tile's rows see; a search over
// their values there (two instructions a word) finds when.  (Brought back at once, the branch
// took so many registers from the loop that some of them went to memory, and each of those
// back behind the copies in flight.)
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
// (o: 16 dims of which v holds eight keys a lane; ones: the row's keys.  One kind after the
// other: beside a tile's registers there is room for no more.)
__device__ __forceinline__ void put_not_finite(const u32x4& v, bf16x8 ones, f32x4& o) {
  auto halves = [](uint32_t bits) { return (bits & 0x00010001u) * 0xFFFFu; };  // of bits 0 and 16
  auto odd = [&](uint32_t x) { return halves(((x & 0x7F807F80u) + 0x00800080u) >> 15); };
  auto fraction = [&](uint32_t x) { return halves(((x & 0x007F007Fu) + 0x007F007Fu) >> 7); };
  auto minus = [&](uint32_t x) { return halves(x >> 15); };
  auto add = [&](auto is, uint32_t value) {
    __builtin_amdgcn_sched_barrier(0);
    u32x4 at;
#pragma unroll
    for (int i = 0; i < 4; i++) at[i] = odd(v[i]) & is(v[i]) & 0x3F803F80u;
    const f32x4 n = mfma16(as_bf16x8(at), ones, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int i = 0; i < 4; i++)  // (n > 0, as a mask)
      o[i] += __uint_as_float((uint32_t)((int)(0u - __float_as_uint(n[i])) >> 31) & value);
  };
  add([&](uint32_t x) { return ~fraction(x) & ~minus(x); }, 0x7F800000u);
  add([&](uint32_t x) { return ~fraction(x) & minus(x); }, 0xFF800000u);
  add([&](uint32_t x) { return fraction(x); }, 0x7FC00000u);
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void drop_not_finite(u32x4& v) {
#pragma unroll
  for (int i = 0; i < 4; i++)
    v[i] &= ~(((((v[i] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu);
}

// Page ids through the constant address space: uniform reads of tables that nothing writes
// during the launch, so they are scalar loads.
typedef const __attribute__((address_space(4))) int32_t* ConstInts;

// An item's rows by their place in it: the token, counted from the first row's, and the q head.
struct ItemRows {
  int rest, group;
  uint32_t inv;
  __device__ __forceinline__ ItemRows(const SpanParams& p, const SpanItem& it)
      : rest(it.rest), group(p.a.group), inv(p.group_inv) {}
  __device__ __forceinline__ int token(int i) const {  // (exact for rest + i < 2^16)
    return group == 1 ? i : (int)__umulhi((unsigned)(rest + i), inv);
  }
  __device__ __forceinline__ int head(int i, int token) const { return rest + i - token * group; }
};
// A row's place in the batch.
struct RowAt {
  int64_t tok;
  int head, pos;
};
__device__ __forceinline__ RowAt row_at(const SpanParams& p, const SpanItem& it, int kvh, int i) {
  const ItemRows rows(p, it);
  const int t = rows.token(i), h = kvh * p.a.group + rows.head(i, t);
  if (it.list) return RowAt{p.tokens[it.tok + t], h, it.pos};
  return RowAt{it.tok + t, h, it.pos + t};
}
// The partial of the item's first row.
__device__ __forceinline__ int64_t part_of(const SpanItem& it, int kvh) {
  return it.part + (int64_t)kvh * it.kvh_stride;
}

// The values of pages v and v + 1 from memory, once more, as a value product takes them: put(e,
// the lane's eight of dim row 16 e + col).
template <int HD, typename Put>
__device__ __forceinline__ void put_back(const SpanParams& p, const Span& span, int kvh, const int32_t* ptab,
                                         int v, int col, int g4, Put&& put) {
  const int64_t page = ptab[span.entry(min(v + (g4 >> 1), span.page_end - 1))];
  const uint16_t* at = p.a.v_pool + (page * p.a.nkv + kvh) * (16 * HD) + col * 16 + 8 * (g4 & 1);
#pragma unroll
  for (int e = 0; e < HD / 16; e++) put(e, *reinterpret_cast<const u32x4*>(at + e * 256));
}

static_assert(kSpanTileRows == 4 * 32, "four waves of two 16-row blocks");
// Tile: 128 rows, 32 of each wave in two blocks of 16, over 32-key chunks that the four
// waves share through LDS, as the bf16 attention's prefill tiles (prefill_item there tells
// how the copies run three chunks ahead).  Chunks that all rows of the tile see whole, from
// first_whole to end_whole, take no masks; those before (the window's low edge, sinks) and
// behind (the diagonal, the end) do, and a wave leaves out those that none of its rows sees.
//
// Bound by the matrix cores and the vector instructions of the softmax beside them.  A whole
// chunk takes 0.7 to 0.8 us with two workgroups on a CU and 0.59 with one, a chunk with masks
// 1.0 to 1.3 at the diagonal and 1.6 to 1.9 at the window's low edge, the start 4 to 5 and the
// end 2.2.  2048 tokens of 64 q heads through a window of 4096 take 247 us, 1.13 PFLOP/s of
// what the rows see, with the matrix cores busy 56% of the time at 1.94 GHz, which the power
// limit leaves.  A prompt of 8191 on 32 heads through 1024 takes 175, 0.74 PFLOP/s of what
// they see, with them busy 33% at 2.26 GHz: half of a tile's 39 us is its start, its end and
// nine chunks of 36 with masks.  128 rows: twice as many in a workgroup would leave one of
// them on a CU, and half as many copy twice as much.  The 32x32x16 instruction takes half the
// issue slots and 290 us where this took 255: the clock falls.
template <int HD>
__device__ __forceinline__ void tile_item(const SpanParams& p, const SpanItem& it, int kvh, char* smem) {
  using SC = SharedChunk<HD>;
  constexpr int KB = SC::KBYTES, CB = SC::BYTES, NLD = SC::NLD, ND = HD / 32;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // row of this lane within each block
  const int g4 = lane >> 4;   // lane group
  const Span span(p, it);
  const ItemRows rows(p, it);
  const int n_rows = it.n_rows;
  const int row0 = 32 * wave;  // the wave's first row, of the item's
  const int first_page = it.page0, page_end = it.page1;
  const int n_chunks = (page_end - first_page + 1) / 2;

  RowState r1 = span_row_start(), r2 = span_row_start();
  const float scale = p.a.scale_log2, inv_scale = 1.f / scale;
  f32x4 o[HD / 16], o2[HD / 16];
#pragma unroll
  for (int db = 0; db < HD / 16; db++) o[db] = o2[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  // positions of the tile's rows and of the wave's
  auto pos_of = [&](int row) {
    return it.list ? it.pos : it.pos + rows.token(min(row, n_rows - 1));
  };
  const int tile_pos0 = pos_of(0), tile_pos1 = pos_of(n_rows - 1);
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

  const ConstInts ptab = (ConstInts)(p.a.pages + it.pages);
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
  int ua, fa = 0;  // page of the chunk the next copy is for, and of the one after
  {
    const int a0 = page_of(0), a1 = page_of(1), a2 = page_of(2);
    ua = page_of(3);
    copy(0, a0);
    copy(1, a1);
    copy(2, a2);
  }
  // the rows' queries, behind the first copies
  bf16x8 qf[ND], qf2[ND];
  int pos, pos2;
  {
    auto load = [&](int row, bf16x8 (&f)[ND], int& at) {
      const RowAt r = row_at(p, it, kvh, min(row, n_rows - 1));
      const uint16_t* qp = p.a.q + r.tok * p.a.q_tok_stride + (int64_t)r.head * HD + 8 * g4;
#pragma unroll
      for (int ds = 0; ds < ND; ds++) f[ds] = as_bf16x8(*reinterpret_cast<const u32x4*>(qp + ds * 32));
      at = r.pos;
    };
    load(row0 + col, qf, pos);
    load(row0 + 16 + col, qf2, pos2);
    // (waited for here: their first use is in loops, where the wait would stay, and would
    // hold for the copies in flight too)
#pragma unroll
    for (int ds = 0; ds < ND; ds++) asm volatile("" : "+v"(qf[ds]), "+v"(qf2[ds]), "+v"(pos), "+v"(pos2));
  }
  const int key0 = 16 * (col >> 3) + 8 * ((col >> 2) & 1) + (col & 3);
  unsigned kaddr[ND];
#pragma unroll
  for (int ds = 0; ds < ND; ds++)
    kaddr[ds] = lds0 + (unsigned)(key0 * (HD * 2) + (((4 * ds + g4) ^ ksw<HD>(key0)) << 4));
  const unsigned vaddr = lds0 + (unsigned)(KB + (g4 >> 1) * (HD * 32) + col * 32 + ((g4 & 1) << 4));

  // Fragments of chunk c (slot: c % 4 as a constant, which then is part of the read
  // instructions, or -1): its keys' score blocks, its values' dims in two halves.
  u32x4 k0[ND], k1[ND];
  auto read_keys = [&](auto slot, int c) {
    constexpr int S = decltype(slot)::value, OFF = S >= 0 ? S * CB : 0;
    const unsigned sb = S >= 0 ? 0u : (unsigned)((c & 3) * CB);
#pragma unroll
    for (int ds = 0; ds < ND; ds++) k0[ds] = lds_read16_at<OFF>(sb + kaddr[ds]);
#pragma unroll
    for (int ds = 0; ds < ND; ds++) k1[ds] = lds_read16_at<OFF + 4 * HD * 2>(sb + kaddr[ds]);
  };
  auto read_values = [&](auto slot, auto half, int c, u32x4 (&v)[ND]) {
    constexpr int S = decltype(slot)::value, OFF = S >= 0 ? S * CB : 0;
    lds_read_run<0, ND, OFF + decltype(half)::value * ND * 512, 512>(
        S >= 0 ? vaddr : vaddr + (unsigned)((c & 3) * CB), v);
  };
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;

  // this lane's raw scores of a chunk, their max, and whether some lane of the wave is above
  // its row's threshold
  float sv1[2][4], sv2[2][4], mx1 = -kInf, mx2 = -kInf;
  auto take = [&](auto mask, const f32x4 (&s1)[2], const f32x4 (&s2)[2], int c) -> bool {
    if constexpr (decltype(mask)::value) {
      mx1 = mask_scores(s1, sv1, seen_keys(span, first_page + 2 * c, pos, g4));
      mx2 = mask_scores(s2, sv2, seen_keys(span, first_page + 2 * c, pos2, g4));
    } else {
      mx1 = take_scores(s1, sv1);
      mx2 = take_scores(s2, sv2);
    }
    return __any(mx1 > r1.thr || mx2 > r2.thr) != 0;
  };
  // (of the wave's rows: fewer chunks need masks than of the tile's)
  auto whole = [&](int c) { return span.all_seen(first_page + 2 * c, wave_pos0, wave_pos1); };
  auto scores = [&](int c) -> bool {  // of a chunk on its own
    read_keys(std::integral_constant<int, -1>{}, c);
    lgkm_wait<0>();
    pin(k0);
    pin(k1);
    const f32x4 s1[2] = {score_block<HD>(k0, qf), score_block<HD>(k1, qf)};
    const f32x4 s2[2] = {score_block<HD>(k0, qf2), score_block<HD>(k1, qf2)};
    if (whole(c)) return take(std::integral_constant<bool, false>{}, s1, s2, c);
    return take(std::integral_constant<bool, true>{}, s1, s2, c);
  };
  const uint32_t no_mask[4] = {};
  auto add_values = [&](auto half, const u32x4 (&v)[ND], bf16x8 pb1, bf16x8 pb2) {
    constexpr int DB0 = decltype(half)::value * ND;
    values_part<HD, DB0, ND, false>(v, o, pb1, no_mask);
    values_part<HD, DB0, ND, false>(v, o2, pb2, no_mask);
  };
  // the values of a chunk that not every row sees whole (no branch may come between a read
  // and its wait); some that are no numbers are left out until the end
  bool left_out = false;
  auto edge_values = [&](int c, bf16x8 pb1, bf16x8 pb2) {
    u32x4 v0[ND], v1[ND];
    read_values(std::integral_constant<int, -1>{}, First{}, c, v0);
    read_values(std::integral_constant<int, -1>{}, Second{}, c, v1);
    lgkm_wait<0>();
    pin(v0);
    pin(v1);
    bool some = false;
    if (!whole(c)) {
#pragma unroll
      for (int e = 0; e < ND; e++) some |= some_not_finite(v0[e]) || some_not_finite(v1[e]);
    }
    if (__any(some)) {
      left_out = true;
#pragma unroll
      for (int e = 0; e < ND; e++) {
        drop_not_finite(v0[e]);
        drop_not_finite(v1[e]);
      }
    }
    add_values(First{}, v0, pb1, pb2);
    add_values(Second{}, v1, pb1, pb2);
  };
  auto raise_rows = [&]() {
    raise_max(r1, mx1, scale, inv_scale, o);
    raise_max(r2, mx2, scale, inv_scale, o2);
  };
  // Top of iteration kt: this wave's copies of chunk kt + 1 have landed, then everyone's, and
  // every read of chunk kt - 1 is done; chunk kt + 3 goes out.  Scalar loads return in any
  // order, so a use of the last iteration's page id behind the issue of the next would wait
  // for that too: the empty statement takes it first.
  auto wait_top = [&](int& use) {
    vm_wait<NLD>();
    asm volatile("" : "+s"(use));
    wg_barrier();
  };
  auto copy_top = [&](int kt, int use, int& fill) {
    fill = page_of(kt + 4);
    copy(kt + 3, use);
  };
  auto run = [&](int kt0, int kt1, auto body) {  // iterations kt0 .. kt1 - 1
    for (int kt = kt0; kt < kt1; kt++) {
      wait_top(ua);
      copy_top(kt, ua, fa);
      body(kt);
      ua = fa;
    }
  };

  if (row0 >= n_rows) {
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
  if (takes(0) && scores(0)) raise_rows();

  // Iteration kt holds the scores of chunk kt (of the previous iteration) and takes its
  // softmax, its values and the scores of chunk kt + 1.
  auto edge = [&](int kt) {
    if (takes(kt)) {
      const bf16x8 pb1 = probs(sv1, r1, scale);
      const bf16x8 pb2 = probs(sv2, r2, scale);
      edge_values(kt, pb1, pb2);
    }
    if (takes(kt + 1) && scores(kt + 1)) raise_rows();
  };
  // The same without masks, where both chunks are whole: the keys of chunk kt + 1 are on
  // their way from LDS during the exponentials of chunk kt, the values of chunk kt during
  // the score products.  slot: kt % 4, or -1.
  auto step = [&](auto slot, int kt, int& use, int& fill) {
    constexpr int S = decltype(slot)::value, S1 = S < 0 ? -1 : (S + 1) % 4;
    wait_top(use);
    read_keys(std::integral_constant<int, S1>{}, kt + 1);
    __builtin_amdgcn_sched_barrier(0);
    copy_top(kt, use, fill);
    const bf16x8 pb1 = probs(sv1, r1, scale);
    const bf16x8 pb2 = probs(sv2, r2, scale);
    u32x4 v0[ND], v1[ND];
    f32x4 s1[2], s2[2];
    lgkm_wait<ND>();
    pin(k0);
    s1[0] = score_block<HD>(k0, qf);
    s2[0] = score_block<HD>(k0, qf2);
    __builtin_amdgcn_sched_barrier(0);  // these products go before the next wait
    read_values(slot, First{}, kt, v0);
    lgkm_wait<ND>();
    pin(k1);
    s1[1] = score_block<HD>(k1, qf);
    s2[1] = score_block<HD>(k1, qf2);
    __builtin_amdgcn_sched_barrier(0);
    read_values(slot, Second{}, kt, v1);
    lgkm_wait<ND>();
    pin(v0);
    add_values(First{}, v0, pb1, pb2);
    const bool raise = take(std::integral_constant<bool, false>{}, s1, s2, kt + 1);
    __builtin_amdgcn_sched_barrier(0);
    lgkm_wait<0>();
    pin(v1);
    add_values(Second{}, v1, pb1, pb2);
    if (raise) raise_rows();
  };
  // the whole chunks' iterations: both kt and kt + 1 are whole, from a multiple of four on
  // four at a time, whose ring slots are constants in the fragment reads
  const int main0 = first_whole, main1 = max(end_whole - 1, main0);
  const int four0 = min((main0 + 3) & ~3, main1), four1 = four0 + ((main1 - four0) & ~3);
  using AnySlot = std::integral_constant<int, -1>;
  auto steps = [&](int kt0, int kt1) {
    for (int kt = kt0; kt < kt1; kt++) {
      step(AnySlot{}, kt, ua, fa);
      ua = fa;
    }
  };
  run(0, main0, edge);
  steps(main0, four0);
  for (int kt = four0; kt < four1; kt += 4) {
    step(std::integral_constant<int, 0>{}, kt, ua, fa);
    step(std::integral_constant<int, 1>{}, kt + 1, fa, ua);
    step(std::integral_constant<int, 2>{}, kt + 2, ua, fa);
    step(std::integral_constant<int, 3>{}, kt + 3, fa, ua);
  }
  steps(four1, main1);
  run(main1, n_chunks, edge);
  vm_wait<0>();  // no copy may land in LDS after the workgroup has ended
  if (left_out) {  // (of the wave) their values once more, from memory
    for (int c = 0; c < n_chunks; c++) {
      if (c == main0) c = main1;
      if (!takes(c)) continue;
      const int v0 = first_page + 2 * c;
      const bf16x8 ones1 = seen_ones(seen_keys(span, v0, pos, g4));
      const bf16x8 ones2 = seen_ones(seen_keys(span, v0, pos2, g4));
      put_back<HD>(p, span, kvh, p.a.pages + it.pages, v0, col, g4, [&](int e, const u32x4& x) {
        put_not_finite(x, ones1, o[e]);
        put_not_finite(x, ones2, o2[e]);
      });
    }
  }

  // the rows' sums over their four lane groups (every lane takes part)
  const float l1 = lane_groups_sum(r1.l), l2 = lane_groups_sum(r2.l);
  const int64_t step32 = p.a.out_tiled ? 512 : 32;
  auto store = [&](int row, float l, const RowState& st, const f32x4 (&acc)[HD / 16]) {
    if (row >= n_rows) return;
    if (it.part >= 0) {
      const int64_t part = part_of(it, kvh) + row;
#pragma unroll
      for (int db = 0; db < HD / 16; db++)
        *reinterpret_cast<f32x4*>(p.a.part_o + part * HD + 16 * db + 4 * g4) = acc[db];
      if (g4 == 0) *reinterpret_cast<float2*>(p.a.part_ml + 2 * part) = float2{st.m, l};
      return;
    }
    const RowAt r = row_at(p, it, kvh, row);
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

// Stream: up to 16 rows (a decode's q heads, a few tokens of a prompt, rows that see a whole
// run); its waves stride over the item's 32-key chunks, keys and values straight to
// registers, and combine through LDS.  Values that no row sees are taken out by select, so
// what their slots hold stays out; those that are no numbers and that some rows see only
// come back at the end, as in a tile.  Keys and values are loaded non-temporally, also beside
// tiles: a call reads them once, and with the cache full of a layer's other data, which they
// would have to push out, 74 decodes beside a shared run take 98 us so and 140 otherwise, a
// prompt of 1024 tokens beside 64 decodes 78 and 90.
//
// Bound by HBM: 128 decodes of 8 KV heads through a window of 4096 read 2.1 GB in 320 us, 6.6
// TB/s; 64 through 1024 their 267 MB in 45, of which some 4 are the first chain of loads (item,
// page id, keys).  With few items that chain is the time: 4 us.  (Eight waves to a workgroup
// where streams are alone in up to 256: nothing gained over batches drawn at random.)
template <int HD>
__device__ __forceinline__ void stream_item(const SpanParams& p, const SpanItem& it, int kvh, char* smem) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int col = lane & 15;  // row of this lane
  const int g4 = lane >> 4;   // lane group
  const int page_end = it.page1;
  const Span span(p, it);
  const RowAt at = row_at(p, it, kvh, min(col, it.n_rows - 1));
  const int pos0 = it.pos, pos1 = it.list ? it.pos : it.pos + ItemRows(p, it).token(it.n_rows - 1);
  bool left_out = false;
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
  const int32_t* ptab = p.a.pages + it.pages;
  auto pid = [&](int v) { return ptab[span.entry(min(v, page_end - 1))]; };
  auto proc = [&](Chunk<HD>& c, int v) {
    const f32x4 s[2] = {score_block<HD>(c.k[0], qf), score_block<HD>(c.k[1], qf)};
    float sv[2][4];
    float mx = take_scores(s, sv);
    if (!span.all_seen(v, pos0, pos1)) {
      mx = mask_scores(s, sv, seen_keys(span, v, at.pos, g4));
      uint32_t keep[4];
      value_mask(seen_keys(span, v, pos0, pos1, g4), keep);
      bool some = false;
#pragma unroll
      for (int db = 0; db < HD / 16; db++) {
#pragma unroll
        for (int h = 0; h < 4; h++) c.v[db][h] &= keep[h];
        some |= some_not_finite(c.v[db]);
      }
      if (pos0 != pos1 && __any(some)) {
        left_out = true;
#pragma unroll
        for (int db = 0; db < HD / 16; db++) drop_not_finite(c.v[db]);
      }
    }
    if (__any(mx > r.thr)) raise_max(r, mx, scale, inv_scale, o);
    const bf16x8 pb = probs(sv, r, scale);
    const uint32_t none[4] = {};
    values_part<HD, 0, HD / 16, false>(c.v, o, pb, none);
  };
  // two chunk buffers in turn, a chunk's loads issued only where it exists (decode_item of
  // the bf16 attention tells why)
  constexpr int STEP = 2 * kWaves;
  Chunk<HD> ca, cb;
  int v = it.page0 + 2 * wave;
  if (v < page_end) {
    int n0 = pid(v + STEP), n1 = pid(v + STEP + 1);
    load_chunk<HD, true>(ca, p.a, kvh, pid(v), pid(v + 1), 0, col, g4);
    while (true) {
      int vn = v + STEP;
      if (vn >= page_end) {
        proc(ca, v);
        break;
      }
      int m0 = pid(vn + STEP), m1 = pid(vn + STEP + 1);
      load_chunk<HD, true>(cb, p.a, kvh, n0, n1, 0, col, g4);
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
      load_chunk<HD, true>(ca, p.a, kvh, n0, n1, 0, col, g4);
      proc(cb, v);
      v = vn;
      n0 = m0;
      n1 = m1;
    }
  }

  if (left_out)  // (of the wave) their values once more
    for (int v = it.page0 + 2 * wave; v < page_end; v += STEP)
      if (!span.all_seen(v, pos0, pos1))
        put_back<HD>(p, span, kvh, ptab, v, col, g4, [&](int e, const u32x4& x) {
          put_not_finite(x, seen_ones(seen_keys(span, v, at.pos, g4)), o[e]);
        });
  // (a row's output in SEGS threads of EL dims each)
  constexpr int SEGS = kWaves * 4, EL = HD / SEGS;
  float(*s_o)[16][HD + 4] = reinterpret_cast<float(*)[16][HD + 4]>(smem);
  float(*s_m)[16] = reinterpret_cast<float(*)[16]>(smem + kWaves * 16 * (HD + 4) * 4);
  float(*s_l)[16] = s_m + kWaves;
#pragma unroll
  for (int db = 0; db < HD / 16; db++)
    *reinterpret_cast<f32x4*>(&s_o[wave][col][db * 16 + 4 * g4]) = o[db];
  const float l = lane_groups_sum(r.l);
  if (g4 == 0) {
    s_m[wave][col] = r.m;
    s_l[wave][col] = l;
  }
  __syncthreads();
  const int row = threadIdx.x / SEGS, seg = threadIdx.x % SEGS;
  const int dseg = seg * EL;
  if (row >= it.n_rows) return;
  float M = kLowest;
#pragma unroll
  for (int w = 0; w < kWaves; w++) M = fmaxf(M, s_m[w][row]);
  float wt[kWaves], L = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    wt[w] = exp2f(s_m[w][row] - M);
    L += s_l[w][row] * wt[w];
  }
  float acc[EL];
#pragma unroll
  for (int e = 0; e < EL; e++) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; w++) a += s_o[w][row][dseg + e] * wt[w];
    acc[e] = a;
  }
  if (it.part < 0) {
    const RowAt to = row_at(p, it, kvh, row);
    const float inv = 1.f / L;
    uint16_t* op = out_ptr(p.a, to.tok, to.head * HD + dseg);  // EL dims within a 32-column block
#pragma unroll
    for (int e = 0; e < EL; e += 2)
      *reinterpret_cast<uint32_t*>(op + e) = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
  } else {
    const int64_t part = part_of(it, kvh) + row;
    float* po = p.a.part_o + part * HD + dseg;
#pragma unroll
    for (int e = 0; e < EL; e += 2) *reinterpret_cast<float2*>(po + e) = float2{acc[e], acc[e + 1]};
    if (seg == 0) *reinterpret_cast<float2*>(p.a.part_ml + 2 * part) = float2{M, L};
  }
}

// An item without pages: partials that count as nothing.
template <int HD>
__device__ __forceinline__ void empty_item(const SpanParams& p, const SpanItem& it, int64_t part) {
  for (int i = threadIdx.x; i < it.n_rows * (HD / 4); i += blockDim.x)
    *reinterpret_cast<f32x4*>(p.a.part_o + part * HD + 4 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
  if ((int)threadIdx.x < it.n_rows)
    *reinterpret_cast<float2*>(p.a.part_ml + 2 * (part + threadIdx.x)) = float2{kLowest, 0.f};
}

// The parameters with the metadata's pointers into the argument block.
struct SmallSpan {
  SpanParams p;
  InlineMeta meta;
};
static_assert(sizeof(SmallSpan) <= 4096, "a launch's arguments");
__device__ __forceinline__ SpanParams inline_params(const SmallSpan& s) {
  SpanParams p = s.p;
  constexpr size_t M = offsetof(SmallSpan, meta);
  p.items = inline_meta(M, p.items);
  p.a.pages = inline_meta(M, p.a.pages);
  p.tokens = inline_meta(M, p.tokens);
  p.merge_tokens = inline_meta(M, p.merge_tokens);
  p.sources = inline_meta(M, p.sources);
  return p;
}

template <int HD>
constexpr int combine_bytes() {
  return (kWaves * 16 * (HD + 4) + 2 * kWaves * 16) * 4;
}
template <int HD, bool TILES>
constexpr int span_smem() {
  return TILES ? smem_bytes<HD>() : combine_bytes<HD>();
}
template <int HD, bool TILES>
__device__ __forceinline__ void span_item(const SpanParams& p, char* smem) {
  const SpanBlock b = span_block(blockIdx.x, p.n_items, p.a.nkv, p.heads);
  const SpanItem it = p.items[b.item];
  if (it.page0 >= it.page1) {
    empty_item<HD>(p, it, part_of(it, b.kvh));
  } else if constexpr (TILES) {
    if (it.kind == 1) tile_item<HD>(p, it, b.kvh, smem);
    else stream_item<HD>(p, it, b.kvh, smem);
  } else {
    stream_item<HD>(p, it, b.kvh, smem);
  }
}
template <int HD, bool TILES>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void span_attn_kernel(
    SpanParams p) {
  __shared__ __attribute__((aligned(16))) char smem[span_smem<HD, TILES>()];
  span_item<HD, TILES>(p, smem);
}
template <int HD, bool TILES>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void small_span_kernel(
    SmallSpan s) {
  __shared__ __attribute__((aligned(16))) char smem[span_smem<HD, TILES>()];
  span_item<HD, TILES>(inline_params(s), smem);
}

// The merge: HD / 4 threads hold a row; a workgroup takes 8 (HD = 128) or 16 q heads of a
// token, or (WIDE) one q head, whose partials its groups of threads read side by side: with
// more than eight partials a row, read one behind another, their latency is the time (from
// four on: a prompt of 3314 tokens 38.6 us a call for 31.5; from 25 on: three decodes of a run
// of 361 pages 34.8 for 31.1).  Bound by latency: 4 us, up to 6 for 128 tokens of 64 q heads.
template <int HD, bool WIDE>
__device__ __forceinline__ void span_merge(const SpanParams& p) {
  constexpr int TPR = HD / 4, G = kMergeThreads / TPR;
  const SpanToken tk = p.merge_tokens[blockIdx.x];
  const int g = threadIdx.x / TPR, d = 4 * (threadIdx.x % TPR);
  const int h = WIDE ? (int)blockIdx.y : (int)blockIdx.y * G + g;
  if (!WIDE && h >= p.a.nq) return;
  const int kvh = h / p.a.group, in_group = h - kvh * p.a.group;
  float m = kLowest, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  int first = WIDE ? g : 0;  // of the next source's splits
  for (int s = 0; s < tk.n_src; s++) {
    const SpanSource src = p.sources[tk.src + s];
    const int64_t base = src.base + (int64_t)kvh * src.kvh_stride + (int64_t)tk.at * p.a.group + in_group;
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
    const float inv = 1.f / l;
    u32x2 w;
    w[0] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    w[1] = pack_bf16x2(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<u32x2*>(out_ptr(p.a, tk.tok, h * HD + d)) = w;
  }
}
template <int HD, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void span_merge_kernel(SpanParams p) {
  span_merge<HD, WIDE>(p);
}
template <int HD, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void small_span_merge_kernel(SmallSpan s) {
  span_merge<HD, WIDE>(inline_params(s));
}

template <int HD>
hipError_t launch(const SpanParams& p, const InlineMeta* meta, bool tiles, int n_merge, int most_parts,
                  hipStream_t stream) {
  const int n = p.n_items * p.a.nkv;
  if (n == 0) return hipSuccess;
  if (meta) {
    const SmallSpan s{p, *meta};
    if (tiles) small_span_kernel<HD, true><<<n, 64 * kWaves, 0, stream>>>(s);
    else small_span_kernel<HD, false><<<n, 64 * kWaves, 0, stream>>>(s);
  } else {
    if (tiles) span_attn_kernel<HD, true><<<n, 64 * kWaves, 0, stream>>>(p);
    else span_attn_kernel<HD, false><<<n, 64 * kWaves, 0, stream>>>(p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || n_merge == 0) return e;
  constexpr int G = kMergeThreads / (HD / 4);
  const bool wide = most_parts > 8;
  const dim3 grid(n_merge, wide ? p.a.nq : (p.a.nq + G - 1) / G);
  if (meta) {
    const SmallSpan s{p, *meta};
    if (wide) small_span_merge_kernel<HD, true><<<grid, kMergeThreads, 0, stream>>>(s);
    else small_span_merge_kernel<HD, false><<<grid, kMergeThreads, 0, stream>>>(s);
  } else {
    if (wide) span_merge_kernel<HD, true><<<grid, kMergeThreads, 0, stream>>>(p);
    else span_merge_kernel<HD, false><<<grid, kMergeThreads, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_span_attn(const SpanParams& p, const InlineMeta* meta, bool tiles, int n_merge,
                            int most_parts, int head_dim, hipStream_t stream) {
  const auto call = head_dim == 128 ? launch<128> : launch<64>;
  return call(p, meta, tiles, n_merge, most_parts, stream);
}

}  // namespace mx
