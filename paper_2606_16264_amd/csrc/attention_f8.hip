// attention_f8.hip -- paged varlen attention over the 8-bit cache for a mixed
// prefill/decode batch on gfx950, and the accumulation of the attention weight of
// every cached token.
//
// The cache holds e4m3 codes and a power-of-two scale per page and KV head.  The
// conversion to bf16 takes the scale as an operand and is exact (a code has four
// significant bits), so from there on this is the bf16 attention: S^T = K Q^T with
// the 16x16x32 bf16 matrix-core instruction, the softmax of a query row held by the
// four lanes l, l ^ 16, l ^ 32, l ^ 48, then O^T += V^T P^T from registers.
//
// The score products are exact and added in fp32.  (The 16x16x128 fp8 instruction on the
// codes as they are, the query as two codes per element, takes 454 instead of 494 us for
// a chunk of 2048 tokens over 14336 of the 8B heads.  But it aligns its products to the
// largest before it adds them, so a score's error grows with sum |q k|: where channels of
// 960 cancel the output was off by 1.6%, where they are 250 by 0.4, and with these
// products by 0.22 in both.)
//
// Keys are consumed four pages (64 keys) at a time.  Score block b, row m is the key
//   kappa_b(m) = token 4 b + m % 4 of page m / 4,
// so that lane group g (rows 4 g .. 4 g + 3 of the four blocks) ends up with the 16
// tokens of page g: one scale per lane for its values, and the tokens of a value
// row of that page are one 16-byte run, in the order the second product takes them.
#include <type_traits>

#include "attention_tile.h"

namespace mx {

namespace {

// Eight codes times a power of two as bf16 (exact).  The instruction reads the
// scale's exponent only.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b, float scale) {
  const mx_bf16x2 w0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
  const mx_bf16x2 w1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const mx_bf16x2 w2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const mx_bf16x2 w3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, w0), __builtin_bit_cast(uint32_t, w1),
                         __builtin_bit_cast(uint32_t, w2), __builtin_bit_cast(uint32_t, w3)});
}

template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint8_t* ptr) {
  const u32x4* q = reinterpret_cast<const u32x4*>(ptr);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  else return *q;
}

// This lane's part of a query row as the first product's B operands: 8 dims
// 64 h + 16 g4 + 8 i .. + 7 for product 2 h + i, as the key codes lie in the lane.
template <int HD>
__device__ __forceinline__ void load_q(const AttnF8Params& p, int64_t tok, int qhead, bool valid,
                                       int g4, bf16x8 (&qf)[HD / 32]) {
  const uint16_t* qp = p.a.q + tok * p.a.q_tok_stride + (int64_t)qhead * HD + 16 * g4;
#pragma unroll
  for (int e = 0; e < HD / 32; e++) {
    const u32x4 v = valid ? *reinterpret_cast<const u32x4*>(qp + 64 * (e >> 1) + 8 * (e & 1))
                          : u32x4{0, 0, 0, 0};
    qf[e] = as_bf16x8(v);
  }
}

// Score block of S^T = K Q^T (16 keys x 16 rows).
template <int HD>
__device__ __forceinline__ f32x4 score_block(const u32x4 (&k)[HD / 64], float ks,
                                             const bf16x8 (&qf)[HD / 32]) {
  f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int h = 0; h < HD / 64; h++) {
    s = mfma16(widen(k[h][0], k[h][1], ks), qf[2 * h], s);
    s = mfma16(widen(k[h][2], k[h][3], ks), qf[2 * h + 1], s);
  }
  return s;
}

// Keys past the range or after the row's position: their scores become kNegBig.
__device__ __forceinline__ void mask_scores(f32x4 (&s)[4], int page, int page_end, int row_pos) {
  const int n = page < page_end ? row_pos - page * 16 : -1;  // the page's last key that counts
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) s[b][i] = 4 * b + i <= n ? s[b][i] : kNegBig;
}
__device__ __forceinline__ float scores_max(const f32x4 (&s)[4]) {
  float mx = kNegBig;
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) mx = fmaxf(mx, s[b][i]);
  return mx;
}

// The step's probabilities of this lane's keys, exp2(score * scale - m), as the
// B operands of the value products (product i: tokens 8 i .. 8 i + 7 of the lane's
// page), and their sum into the lane's share of the row's sum: from the rounded
// values that the products use, or (EXACT) from the values before that rounding,
// which the accumulated weights need: theirs is an fp32 result, and the rounded
// sum of a row is off by up to 2^-9.
template <bool EXACT>
__device__ __forceinline__ bf16x8 half_probs(const f32x4& s0, const f32x4& s1, RowState& r,
                                             float scale_log2) {
  const mx_bf16x2 ones = __builtin_bit_cast(mx_bf16x2, 0x3F803F80u);
  float pv[2][4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    pv[0][i] = fast_exp2(fmaf(s0[i], scale_log2, -r.m));
    pv[1][i] = fast_exp2(fmaf(s1[i], scale_log2, -r.m));
  }
  const uint32_t w0 = pack_bf16x2(pv[0][0], pv[0][1]);
  const uint32_t w1 = pack_bf16x2(pv[0][2], pv[0][3]);
  const uint32_t w2 = pack_bf16x2(pv[1][0], pv[1][1]);
  const uint32_t w3 = pack_bf16x2(pv[1][2], pv[1][3]);
  if constexpr (EXACT) {
    r.l += ((pv[0][0] + pv[0][1]) + (pv[0][2] + pv[0][3])) +
           ((pv[1][0] + pv[1][1]) + (pv[1][2] + pv[1][3]));
  } else {
    r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w0), ones, r.l, false);
    r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w1), ones, r.l, false);
    r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w2), ones, r.l, false);
    r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w3), ones, r.l, false);
  }
  return as_bf16x8(u32x4{w0, w1, w2, w3});
}
template <bool EXACT>
__device__ __forceinline__ void probs(const f32x4 (&s)[4], RowState& r, float scale_log2,
                                      bf16x8 (&pb)[2]) {
  pb[0] = half_probs<EXACT>(s[0], s[1], r, scale_log2);
  pb[1] = half_probs<EXACT>(s[2], s[3], r, scale_log2);
}

// Which of the 16 tokens of this lane's value page hold values (bytes of a value
// row): tokens past the request's length are zeroed by select, not multiplied, so
// that NaN codes left there stay out of the sum.
__device__ __forceinline__ void value_keep(int page, int page_end, int kv_len,
                                           uint32_t (&keep)[4]) {
  const int n = page < page_end ? min(max(kv_len - page * 16, 0), 16) : 0;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const int b = min(max(n - 4 * w, 0), 4);
    keep[w] = b == 4 ? ~0u : (1u << (8 * b)) - 1;
  }
}

// O^T += V^T P^T over the output blocks DB0 .. DB0 + NDB - 1 (16 head dims each).
template <int HD, int DB0, int NDB>
__device__ __forceinline__ void values_part(const u32x4 (&v)[NDB], float vs, f32x4 (&o)[HD / 16],
                                            const bf16x8 (&pb)[2]) {
#pragma unroll
  for (int e = 0; e < NDB; e++) {
    o[DB0 + e] = mfma16(widen(v[e][0], v[e][1], vs), pb[0], o[DB0 + e]);
    o[DB0 + e] = mfma16(widen(v[e][2], v[e][3], vs), pb[1], o[DB0 + e]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The scan of a decode: the wave's 64-key steps at pages pi, pi + 16 .. below
// page_end.  One register buffer for the keys of a step and one for its values, each
// filled again for the next step as soon as its products have been taken: the next
// keys are in flight during the softmax and the value products, the next values
// during the next score products.  (Two buffers of both, in turn, took more than the
// 256 registers of a wave, and a spilled register comes back behind every load in
// flight: 256 decodes of the 8B heads 651 us.)  Only a wave's last step can hold keys
// that do not count.  The loads are unconditional on every path, so that the waits
// cover exactly what they need.
template <int HD, bool NT, bool TRACK>
struct DecodeScan {
  const AttnF8Params& p;
  const int32_t* ptab;
  int kvh, page_end, row_pos, kv_len, col, g4;
  float scale, inv_scale;
  float* scores;  // TRACK: where the lane leaves scores in log2 units (store_scores), or null
  int rows;       // TRACK: 4, 8 or 16, at least the item's rows
  u32x4 k[4][HD / 64], v[HD / 16];
  float ks, vs;

  // the lane's key and value pages (past the range: its last page, masked there)
  __device__ __forceinline__ int key_page(int pi) const { return ptab[min(pi + (col >> 2), page_end - 1)]; }
  __device__ __forceinline__ int value_page(int pi) const { return ptab[min(pi + g4, page_end - 1)]; }
  __device__ __forceinline__ void load_keys(int page) {
    const int64_t at = (int64_t)page * p.a.nkv + kvh;
    const uint8_t* src = p.k8 + at * (16 * HD) + (col & 3) * 64 + 16 * g4;
    ks = p.k_scale[at];
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int h = 0; h < HD / 64; h++) k[b][h] = load16<NT>(src + h * 1024 + b * 256);
  }
  __device__ __forceinline__ void load_values(int page) {
    const int64_t at = (int64_t)page * p.a.nkv + kvh;
    const uint8_t* src = p.v8 + at * (16 * HD) + col * 16;
    vs = p.v_scale[at];
#pragma unroll
    for (int db = 0; db < HD / 16; db++) v[db] = load16<true>(src + db * 256);
  }
  __device__ __forceinline__ void score(const bf16x8 (&qf)[HD / 32], f32x4 (&s)[4]) {
#pragma unroll
    for (int b = 0; b < 4; b++) {
      s[b] = score_block<HD>(k[b], ks, qf);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The scores of the item's rows, 64 bytes a row and page.  With up to 4 (8) rows the
  // lanes of the other columns take blocks 1 .. 3 (the odd blocks) of those rows, so
  // that one store (two) holds whole runs and not a quarter of each with a quarter of
  // the lanes: 64 decodes of the 8B heads 108 -> 101 us (82 without weights).
  __device__ __forceinline__ void store_scores(const f32x4 (&s)[4], int pi, bool valid) {
    auto moved = [&](float to, float from, auto ctrl, auto banks) {  // banks: columns / 4
      return __uint_as_float(__builtin_amdgcn_update_dpp(
          (int)__float_as_uint(to), (int)__float_as_uint(from), decltype(ctrl)::value, 0xF,
          decltype(banks)::value, false));
    };
    using std::integral_constant;
    f32x4* out = reinterpret_cast<f32x4*>(scores + pi * 16);
    const bool store = scores && valid;
    if (rows == 4) {
      f32x4 x;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        x[i] = moved(s[0][i], s[1][i], integral_constant<int, 0x114>{}, integral_constant<int, 2>{});
        x[i] = moved(x[i], s[2][i], integral_constant<int, 0x118>{}, integral_constant<int, 4>{});
        x[i] = moved(x[i], s[3][i], integral_constant<int, 0x11C>{}, integral_constant<int, 8>{});
      }
      if (store) *out = x * scale;
    } else if (rows == 8) {
      f32x4 x, y;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        x[i] = moved(s[0][i], s[1][i], integral_constant<int, 0x118>{}, integral_constant<int, 12>{});
        y[i] = moved(s[2][i], s[3][i], integral_constant<int, 0x118>{}, integral_constant<int, 12>{});
      }
      if (store) {
        out[0] = x * scale;
        out[2] = y * scale;
      }
    } else if (store) {
#pragma unroll
      for (int b = 0; b < 4; b++) out[b] = s[b] * scale;
    }
  }
  template <bool LAST>
  __device__ __forceinline__ void softmax(f32x4 (&s)[4], int pi, RowState& r, f32x4 (&o)[HD / 16],
                                          bf16x8 (&pb)[2]) {
    const int page = pi + g4;
    if constexpr (LAST) mask_scores(s, page, page_end, row_pos);
    if constexpr (TRACK) store_scores(s, pi, !LAST || page < page_end);
    const float mx = scores_max(s);
    if (__any(mx > r.thr)) raise_max(r, mx, scale, inv_scale, o);
    probs<TRACK>(s, r, scale, pb);
  }
  __device__ __forceinline__ void run(int pi, const bf16x8 (&qf)[HD / 32], f32x4 (&o)[HD / 16],
                                      RowState& r) {
    if (pi >= page_end) return;
    f32x4 s[4];
    bf16x8 pb[2];
    // The order of the loads is that of their uses, page ids of the next step first, on
    // every way into the loop: a wait counts what was issued behind the load it is for,
    // and takes the least count of all ways.
    const int k0 = key_page(pi), v0 = value_page(pi);
    int kn = key_page(pi + 16), vn = value_page(pi + 16);
    __builtin_amdgcn_sched_barrier(0);
    load_keys(k0);
    __builtin_amdgcn_sched_barrier(0);
    load_values(v0);
    __builtin_amdgcn_sched_barrier(0);
    for (; pi + 16 < page_end; pi += 16) {
      score(qf, s);
      const int kn2 = key_page(pi + 32), vn2 = value_page(pi + 32);
      __builtin_amdgcn_sched_barrier(0);
      load_keys(kn);
      __builtin_amdgcn_sched_barrier(0);
      softmax<false>(s, pi, r, o, pb);
      values_part<HD, 0, HD / 16>(v, vs, o, pb);
      load_values(vn);
      __builtin_amdgcn_sched_barrier(0);
      kn = kn2;
      vn = vn2;
    }
    score(qf, s);
    softmax<true>(s, pi, r, o, pb);
    uint32_t keep[4];
    value_keep(pi + g4, page_end, kv_len, keep);
#pragma unroll
    for (int db = 0; db < HD / 16; db++)
#pragma unroll
      for (int w = 0; w < 4; w++) v[db][w] &= keep[w];
    values_part<HD, 0, HD / 16>(v, vs, o, pb);
  }
};

// Decode item: the q heads it.head .. it.head + nrows - 1 (one per lane row) of the
// request's single token, over pages it.start .. of its table; the four waves
// stride over the split's 64-key chunks and combine through LDS.
template <int HD, bool NT, bool TRACK>
__device__ __forceinline__ void decode_item(const AttnF8Params& p, const AttnItem& it,
                                            const ReqDev& rq, char* smem) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // q head of this lane (relative to it.head)
  const int g4 = lane >> 4;   // lane group
  const bool row_valid = col < it.nrows;
  const int qhead = it.head + (row_valid ? col : 0);
  const int64_t qtok = rq.tok_start;
  RowState r = row_start();
  f32x4 o[HD / 16];
#pragma unroll
  for (int db = 0; db < HD / 16; db++) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 qf[HD / 32];
  load_q<HD>(p, qtok, qhead, row_valid, g4, qf);
  float* scores = nullptr;
  const int rows = it.nrows <= 4 ? 4 : it.nrows <= 8 ? 8 : 16;
  if constexpr (TRACK) {
    const int r = col & (rows - 1), b = col / rows;  // row and first block of the lane's stores
    if (r < it.nrows)
      scores = p.scores + p.score_base[it.req] + (it.head + r) * score_row(rq.n_pages) + 16 * g4 +
               4 * b;
  }
  DecodeScan<HD, NT, TRACK> scan{p, p.a.pages + rq.page_start, it.head / p.a.group,
                                 min(it.start + p.a.split_pages, rq.n_pages), rq.kv_len - 1,
                                 rq.kv_len, col, g4, p.a.scale_log2, 1.f / p.a.scale_log2, scores,
                                 rows, {}, {}, 0.f, 0.f};
  scan.run(it.start + 4 * wave, qf, o, r);

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
  if (row >= it.nrows) return;
  float M = kNegBig;
#pragma unroll
  for (int w = 0; w < 4; w++) M = fmaxf(M, s_m[w][row]);
  float wt[4], L = 0.f;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    wt[w] = exp2f(s_m[w][row] - M);  // a wave without a key: 0 (the first wave has one)
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
  const int h = it.head + row;
  if (rq.n_split == 1) {
    const float inv = 1.f / L;
    uint16_t* op = out_ptr(p.a, qtok, h * HD + dseg);  // HD / 16 dims within a 32-column block
#pragma unroll
    for (int e = 0; e < HD / 16; e += 2)
      *reinterpret_cast<uint32_t*>(op + e) = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
    if (TRACK && (threadIdx.x & 15) == 0) p.lse[qtok * p.a.nq + h] = M + log2f(L);
  } else {
    const int64_t part = (int64_t)it.part + (int64_t)row * rq.n_split;
    float* po = p.a.part_o + part * HD + dseg;
#pragma unroll
    for (int e = 0; e < HD / 16; e += 4)
      *reinterpret_cast<f32x4*>(po + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
    if ((threadIdx.x & 15) == 0) {
      p.a.part_ml[part * 2 + 0] = M;
      p.a.part_ml[part * 2 + 1] = L;
    }
  }
}

// The top bits of the bytes that hold a NaN (a code of magnitude 0x7F).
__device__ __forceinline__ u32x4 nan_codes(const u32x4& w) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = ((w[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
  return x;
}
// Where rows see some of the keys only and a value is NaN, a probability of 0 would not
// keep it out of their products.  So it is taken out there (by the caller), and what it
// belongs in is found by a product of its own, of the NaNs' places with the keys that the
// lane's row sees (its page's tokens 0 .. last).  The search costs a fresh prompt of 512
// tokens of the 8B heads 0.8 us of 17, one of 2048 1 of 58 (a branch for two blocks at
// a time: no less, and 15 registers spilled where weights are accumulated).
__device__ __forceinline__ void nan_values(const u32x4& nan, int last, f32x4& o) {
  f32x4 seen = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; i++) {
    uint32_t row[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int tok = 8 * i + 2 * e;
      row[e] = (tok <= last ? 0x3F80u : 0u) | (tok < last ? 0x3F800000u : 0u);
    }
    // (0x38: the code of 1.0)
    seen = mfma16(widen((nan[2 * i] >> 7) * 0x38u, (nan[2 * i + 1] >> 7) * 0x38u, 1.f),
                  as_bf16x8(u32x4{row[0], row[1], row[2], row[3]}), seen);
  }
#pragma unroll
  for (int e = 0; e < 4; e++) o[e] = seen[e] > 0.f ? __builtin_nanf("") : o[e];
}

// Prefill tiles share every 64-key chunk through LDS.  Wave w copies page w of the
// chunk there with the DMA path (global_load_lds, 16 bytes per lane): its keys, its
// values and, by an ordinary store, its two scales.  Keys keep the page's layout but
// for the four 16-byte pieces of a 64-byte run, stored at piece i ^ key_swizzle(w): the
// 16 lanes that the LDS serves at a time ({0-3, 12-15, 20-23, 24-27} and so on) then
// hit distinct bank groups, in both pairs of pages that such a set reads.  Values are
// unswizzled: the sets' 16 rows are distinct modulo 16 already.
__device__ __forceinline__ int key_swizzle(int page) { return (4 - page) & 3; }
template <int HD>
struct SharedChunk8 {
  static constexpr int PAGE = 16 * HD;        // bytes of a page's keys (values) of one head
  static constexpr int BYTES = 8 * PAGE;      // a chunk: four pages' keys, then their values
  static constexpr int SLOTS = 4;             // chunks kt .. kt + 3: copies run three ahead
  static constexpr int NLD = 2 * PAGE / 1024; // 1 KB copies per wave per chunk
  static constexpr int SCALES = SLOTS * BYTES;  // [slot][page] (key scale, value scale)
};
template <int HD>
constexpr int smem_bytes() {
  constexpr int ring = SharedChunk8<HD>::SCALES + SharedChunk8<HD>::SLOTS * 4 * 8;
  constexpr int combine = (4 * 16 * (HD + 4) + 2 * 4 * 16) * 4;
  return ring > combine ? ring : combine;
}

// The 4 bytes at LDS address addr + OFF; a pair of words there.
template <int OFF>
__device__ __forceinline__ uint32_t lds_read4_at(unsigned addr) {
  uint32_t v;
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
__device__ __forceinline__ void lds_write8(unsigned addr, u32x2 v) {
  asm volatile("ds_write_b64 %0, %1" ::"v"(addr), "v"(v) : "memory");
}
__device__ __forceinline__ void pin1(uint32_t& x) { asm volatile("" : "+v"(x)); }

// Prefill item: rows it.start .. it.start + 127 of `pack` q heads of one KV head (a power
// of two), row r being q head it.head + r % pack and new token r / pack, so that heads
// which share their keys share a tile; wave w owns two blocks of 16 consecutive rows,
// it.start + 32 w + (0 | 16) + col.  With few tiles over long contexts each is split over
// its keys (choose_tiles): a split takes its chunks as a tile of a shorter request, whose
// positions count from its first key, and leaves unnormalised rows, their maxima and
// sums for merge_tile.
//
// Iteration kt of the chunk loop reads the keys of chunk kt + 1 for the score products
// while the exponentials of chunk kt (whose scores the previous iteration left) run on
// the vector units, then takes the value products of chunk kt, and raises the rows'
// running max for chunk kt + 1 where needed.  The copies of chunk kt + 3 go out at the
// top of iteration kt into the slot chunk kt - 1 used, after the barrier that ends
// every wave's reads of it, and the scales of that chunk's page are read (scalar
// loads) with them and stored to LDS one iteration later.  Every iteration issues the
// same copies (chunks past the tile's last one copy the tile's last page into the free
// slot and are never read), and they are the only vector-memory operations of the
// loop, so one vmcnt value fits every wait: at the top of iteration kt the copies of
// iteration kt - 1 may still be in flight, every earlier one (chunk kt + 1) has landed.
static_assert(kPrefillTileRows == 4 * 32, "four waves of two 16-row blocks");
template <int HD, bool TRACK>
__device__ __forceinline__ void prefill_item(const AttnF8Params& p, const AttnItem& it,
                                             const ReqDev& rq, char* smem) {
  using SC = SharedChunk8<HD>;
  constexpr int CB = SC::BYTES, NLD = SC::NLD, NH = HD / 64;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15;  // query row of this lane within each block
  const int g4 = lane >> 4;   // lane group
  const int kvh = it.head / p.a.group, shift = p.pack_log2, rows = rq.n_new << shift;
  const int n_split = it.nrows, split = it.start % kPrefillTileRows, start = it.start - split;
  const int row0 = start + 32 * wave;
  // the split's chunks: `per` each, as split_tile of the host has it
  int ctx_len = rq.ctx_len, kv_len = rq.kv_len, first_page = 0, most_pages = rq.n_pages;
  if (n_split > 1) {
    const int chunks = (ctx_len + (start >> shift)) / 64 + 1;
    const int per = (chunks + n_split - 1) / n_split;
    ctx_len -= 64 * per * split;
    kv_len -= 64 * per * split;
    first_page = 4 * per * split;
    if (split < n_split - 1) most_pages = 4 * per;
  }
  struct Row {
    int token, head;  // of the chunk's new tokens; q head
    bool valid;
  };
  auto row_at = [&](int r) {
    const int rc = min(r, rows - 1), token = rc >> shift;
    return Row{token, it.head + rc - (token << shift), r < rows};
  };
  auto pages_to = [&](int r) {  // that row r, or the last one, sees
    return min((ctx_len + (min(r, rows - 1) >> shift)) / 16 + 1, most_pages);
  };
  const int page_end = row0 < rows ? pages_to(row0 + 31) : 0;
  const float scale = p.a.scale_log2, inv_scale = 1.f / scale;

  bf16x8 qf[HD / 32], qf2[HD / 32];
  int row_pos, row_pos2;
  {
    const Row a = row_at(row0 + col), b = row_at(row0 + 16 + col);
    load_q<HD>(p, rq.tok_start + a.token, a.head, a.valid, g4, qf);
    load_q<HD>(p, rq.tok_start + b.token, b.head, b.valid, g4, qf2);
    row_pos = ctx_len + a.token;
    row_pos2 = ctx_len + b.token;
  }
  RowState r1 = row_start(), r2 = row_start();
  f32x4 o[HD / 16], o2[HD / 16];
#pragma unroll
  for (int db = 0; db < HD / 16; db++) o[db] = o2[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  // the tile's last row bounds the pages every wave helps to copy
  const int item_pages = pages_to(start + kPrefillTileRows - 1);
  const int n_chunks = (item_pages + 3) / 4;
  const int wave_chunks = (page_end + 3) / 4;  // 0 for a wave without valid rows
  // page ids and scales through the constant address space: uniform reads of tables
  // nothing writes during the launch, so they are scalar loads
  typedef const __attribute__((address_space(4))) int32_t* ConstInts;
  typedef const __attribute__((address_space(4))) float* ConstFloats;
  const ConstInts ptab = (ConstInts)(p.a.pages + rq.page_start + first_page);
  const ConstFloats k_scale = (ConstFloats)p.k_scale, v_scale = (ConstFloats)p.v_scale;

  // byte offsets in the page of this lane's share of a key copy (of 64 dims) and of a
  // value copy: the LDS is written in lane order
  const unsigned k_off = (lane >> 2) * 64 + (((lane & 3) ^ key_swizzle(wave)) << 4);
  const unsigned v_off = lane * 16;
  const unsigned lds0 = (unsigned)(size_t)(MX_LDS char*)smem;
  const unsigned dst0 = lds0 + (unsigned)(wave * SC::PAGE);
  const unsigned scale0 = lds0 + SC::SCALES;
  auto copy = [&](int c, int page) {  // the wave's copies of chunk c
    const int64_t at = ((int64_t)page * p.a.nkv + kvh) * SC::PAGE;
    const uint8_t *kp = p.k8 + at, *vp = p.v8 + at;
    const unsigned dst = dst0 + (unsigned)((c & 3) * CB);
#pragma unroll
    for (int h = 0; h < NH; h++) dma16_at(kp, k_off + 1024 * h, dst + 1024 * h);
#pragma unroll
    for (int h = 0; h < NH; h++) dma16_at(vp, v_off + 1024 * h, dst + 4 * SC::PAGE + 1024 * h);
  };
  struct Scales {
    float k, v;
  };
  auto scales_of = [&](int page) {
    const int64_t at = (int64_t)page * p.a.nkv + kvh;
    return Scales{k_scale[at], v_scale[at]};
  };
  auto put_scales = [&](int c, const Scales& s) {
    if (lane == 0)
      lds_write8(scale0 + (unsigned)((c & 3) * 32 + wave * 8),
                 u32x2{__float_as_uint(s.k), __float_as_uint(s.v)});
  };
  // the page this wave copies of chunk c (past the tile's last page: that page, whose
  // keys are masked there)
  auto page_of = [&](int c) { return ptab[min(4 * c + wave, item_pages - 1)]; };

  // fragment addresses within a slot: score block b of key rows kappa_b(col) is 256
  // bytes after block b - 1, 64 dims are 1 KB; value dim rows 16 e + col of page g4
  const int kpage = col >> 2;
  const unsigned kaddr = lds0 + (unsigned)(kpage * SC::PAGE + (col & 3) * 64 +
                                           ((g4 ^ key_swizzle(kpage)) << 4));
  const unsigned vaddr = lds0 + (unsigned)((4 + g4) * SC::PAGE + col * 16);
  const unsigned ks_addr = scale0 + kpage * 8, vs_addr = scale0 + g4 * 8;

  // (slot: the chunk's ring slot as a constant, which then is part of the read
  // instructions, or -1)
  // raw scores of chunk c from its keys in LDS, their max, and whether some lane of
  // the wave is above its row's threshold; beside(b) goes with the products of block b
  f32x4 s1[4], s2[4];
  float mx1 = kNegBig, mx2 = kNegBig;
  auto scores = [&](auto mask, auto slot, int c, auto beside) -> bool {
    constexpr bool MASK = decltype(mask)::value;
    constexpr int S = decltype(slot)::value, OFF = S >= 0 ? S * CB : 0, SOFF = S >= 0 ? S * 32 : 0;
    const unsigned ka = S >= 0 ? kaddr : kaddr + (unsigned)((c & 3) * CB);
    uint32_t ks = lds_read4_at<SOFF>(S >= 0 ? ks_addr : ks_addr + (unsigned)((c & 3) * 32));
    u32x4 k[4][NH];
    f32x4 n1[4], n2[4];
    auto read = [&](auto b) {
      constexpr int B = decltype(b)::value;
      k[B][0] = lds_read16_at<OFF + B * 256>(ka);
      if constexpr (NH == 2) k[B][1] = lds_read16_at<OFF + B * 256 + 1024>(ka);
    };
    auto block = [&](auto b) {
      constexpr int B = decltype(b)::value;
      lgkm_wait<(3 - B) * NH>();
      if constexpr (B == 0) pin1(ks);
      pin(k[B]);
      n1[B] = n2[B] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < NH; h++)
#pragma unroll
        for (int i = 0; i < 2; i++) {
          const bf16x8 w = widen(k[B][h][2 * i], k[B][h][2 * i + 1], __uint_as_float(ks));
          n1[B] = mfma16(w, qf[2 * h + i], n1[B]);
          n2[B] = mfma16(w, qf2[2 * h + i], n2[B]);
        }
      beside(b);
      __builtin_amdgcn_sched_barrier(0);  // these products go before the next wait
    };
    using std::integral_constant;
    read(integral_constant<int, 0>{});
    read(integral_constant<int, 1>{});
    read(integral_constant<int, 2>{});
    read(integral_constant<int, 3>{});
    block(integral_constant<int, 0>{});
    block(integral_constant<int, 1>{});
    block(integral_constant<int, 2>{});
    block(integral_constant<int, 3>{});
#pragma unroll
    for (int b = 0; b < 4; b++) {
      s1[b] = n1[b];
      s2[b] = n2[b];
    }
    if constexpr (MASK) {
      mask_scores(s1, 4 * c + g4, page_end, row_pos);
      mask_scores(s2, 4 * c + g4, page_end, row_pos2);
    }
    mx1 = scores_max(s1);
    mx2 = scores_max(s2);
    return __any(mx1 > r1.thr || mx2 > r2.thr) != 0;
  };
  auto nothing = [](auto) {};
  // value products of chunk c (values past the request's keys zeroed when MASK: only
  // the chunk that holds the request's last key has such values)
  auto values = [&](auto mask, auto slot, int c, const bf16x8 (&pb1)[2], const bf16x8 (&pb2)[2]) {
    constexpr bool MASK = decltype(mask)::value;
    constexpr int S = decltype(slot)::value, OFF = S >= 0 ? S * CB : 0, SOFF = S >= 0 ? S * 32 : 0;
    constexpr int Q = HD / 64;  // value rows per part: four parts
    const unsigned va = S >= 0 ? vaddr : vaddr + (unsigned)((c & 3) * CB);
    uint32_t vs = lds_read4_at<SOFF + 4>(S >= 0 ? vs_addr : vs_addr + (unsigned)((c & 3) * 32));
    u32x4 v[4][Q];
    lds_read_run<0, Q, OFF, 256>(va, v[0]);
    lds_read_run<0, Q, OFF + Q * 256, 256>(va, v[1]);
    lds_read_run<0, Q, OFF + 2 * Q * 256, 256>(va, v[2]);
    lds_read_run<0, Q, OFF + 3 * Q * 256, 256>(va, v[3]);
    uint32_t keep[4];
    if constexpr (MASK) value_keep(4 * c + g4, page_end, kv_len, keep);
    auto part = [&](auto b) {
      constexpr int B = decltype(b)::value;
      lgkm_wait<(3 - B) * Q>();
      if constexpr (B == 0) pin1(vs);
      pin(v[B]);
#pragma unroll
      for (int e = 0; e < Q; e++) {
        u32x4 w = v[B][e];
        if constexpr (MASK) {
#pragma unroll
          for (int i = 0; i < 4; i++) w[i] &= keep[i];
          const u32x4 nan = nan_codes(w);
          if (__any(((nan[0] | nan[1]) | (nan[2] | nan[3])) != 0)) {
            const int key = (4 * c + g4) * 16;
            nan_values(nan, row_pos - key, o[B * Q + e]);
            nan_values(nan, row_pos2 - key, o2[B * Q + e]);
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] &= ~((nan[i] >> 7) * 0xFFu);
          }
        }
#pragma unroll
        for (int i = 0; i < 2; i++) {
          const bf16x8 f = widen(w[2 * i], w[2 * i + 1], __uint_as_float(vs));
          o[B * Q + e] = mfma16(f, pb1[i], o[B * Q + e]);
          o2[B * Q + e] = mfma16(f, pb2[i], o2[B * Q + e]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // these products go before the next wait
    };
    part(std::integral_constant<int, 0>{});
    part(std::integral_constant<int, 1>{});
    part(std::integral_constant<int, 2>{});
    part(std::integral_constant<int, 3>{});
  };
  auto raise_rows = [&]() {
    raise_max(r1, mx1, scale, inv_scale, o);
    raise_max(r2, mx2, scale, inv_scale, o2);
  };
  using Masked = std::integral_constant<bool, true>;
  using Unmasked = std::integral_constant<bool, false>;

  // prologue: the copies of chunks 0 .. 2, the scales of chunks 0 and 1 in LDS
  int ua, fa = 0;  // page of the chunk the next copy is for, and of the one after
  Scales sc;       // scales of the chunk copied last
  {
    const int a0 = page_of(0), a1 = page_of(1), a2 = page_of(2);
    copy(0, a0);
    copy(1, a1);
    ua = page_of(3);
    copy(2, a2);
    put_scales(0, scales_of(a0));
    put_scales(1, scales_of(a1));
    sc = scales_of(a2);
  }
  // top of iteration kt: this wave's copies of chunk kt + 1 have landed and its scale
  // stores are done, then everyone's, and every read of chunk kt - 1 is done; chunk
  // kt + 3 goes out, the scales of chunk kt + 2 go to LDS.  Scalar loads return in any
  // order, so a use of the last iteration's behind the issue of this one's would wait
  // for those too: the empty statement takes the old ones first.
  auto top = [&](int kt, int& use, int& fill) {
    vm_wait<NLD>();
    lgkm_wait<0>();
    asm volatile("" : "+s"(use), "+s"(sc.k), "+s"(sc.v));
    const Scales old = sc;
    fill = page_of(kt + 4);
    sc = scales_of(use);
    wg_barrier();
    put_scales(kt + 2, old);
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

  // chunk 0 and the first scales have landed; chunks 1 and 2 may be in flight
  vm_wait<2 * NLD>();
  lgkm_wait<0>();
  wg_barrier();
  if (row0 >= rows) {
    // no rows here: this wave only copies its page of every chunk
    run(0, n_chunks, [](int) {});
    vm_wait<0>();  // no copy may land in LDS after the workgroup has ended
    return;
  }
  if (scores(Masked{}, std::integral_constant<int, 0>{}, 0, nothing)) raise_rows();  // the first step raises every row's max

  // Chunks 0 .. n_int - 1 are inside every wave's range and at or before every row of
  // the tile: no masks.  The last chunk of the tile is the only one that can hold keys
  // past the request's end, so n_main <= n_chunks - 1.
  const int first_pos = ctx_len + (start >> shift);
  const int page_end0 = pages_to(start + 31);  // wave 0's
  const int n_int = first_pos >= 63 ? min((first_pos - 63) / 64 + 1, page_end0 / 4) : 0;
  const int n_main = max(0, n_int - 1);
  auto step = [&](auto slot, int kt) {  // slot: kt % 4 or -1
    constexpr int S = decltype(slot)::value, S1 = S < 0 ? -1 : (S + 1) % 4;
    bf16x8 pb1[2], pb2[2];
    const bool raise = scores(Unmasked{}, std::integral_constant<int, S1>{}, kt + 1, [&](auto b) {
      constexpr int B = decltype(b)::value, H = B & 1;
      if constexpr (B < 2) pb1[H] = half_probs<TRACK>(s1[2 * H], s1[2 * H + 1], r1, scale);
      else pb2[H] = half_probs<TRACK>(s2[2 * H], s2[2 * H + 1], r2, scale);
    });
    values(Unmasked{}, slot, kt, pb1, pb2);
    if (raise) raise_rows();
  };
  // four chunks at a time, whose ring slots are constants in the fragment reads
  const int n4 = n_main & ~3;
  for (int kt = 0; kt < n4; kt += 4) {
    top(kt, ua, fa);
    step(std::integral_constant<int, 0>{}, kt);
    top(kt + 1, fa, ua);
    step(std::integral_constant<int, 1>{}, kt + 1);
    top(kt + 2, ua, fa);
    step(std::integral_constant<int, 2>{}, kt + 2);
    top(kt + 3, fa, ua);
    step(std::integral_constant<int, 3>{}, kt + 3);
  }
  using AnySlot = std::integral_constant<int, -1>;
  run(n4, n_main, [&](int kt) { step(AnySlot{}, kt); });
  // the chunks around the diagonal and the tile's end, with masks and bounds
  run(n_main, n_chunks, [&](int kt) {
    const bool more = kt + 1 < wave_chunks;  // scores of chunk kt + 1
    if (kt < wave_chunks) {
      bf16x8 pb1[2], pb2[2];
      probs<TRACK>(s1, r1, scale, pb1);
      probs<TRACK>(s2, r2, scale, pb2);
      values(Masked{}, AnySlot{}, kt, pb1, pb2);
    }
    if (more && scores(Masked{}, AnySlot{}, kt + 1, nothing)) raise_rows();
  });
  vm_wait<0>();  // no copy may land in LDS after the workgroup has ended

  // the rows' sums over their four lane groups (every lane takes part)
  const float l1 = lane_groups_sum(r1.l), l2 = lane_groups_sum(r2.l);
  // dims 16 db + 4 g4 .. + 3 of the row: (db / 2) 32-column steps plus 16 (db % 2)
  const int64_t step32 = p.a.out_tiled ? 512 : 32;
  int end_col = threadIdx.x;  // (the rows once more: kept over the loop they cost registers)
  asm volatile("" : "+v"(end_col));
  end_col &= 15;
  if (n_split > 1) {
    auto leave = [&](int r, float l, const RowState& st, const f32x4 (&acc)[HD / 16]) {
      if (row0 + r >= rows) return;
      const int64_t part = (int64_t)it.part + 32 * wave + r;
#pragma unroll
      for (int db = 0; db < HD / 16; db++)
        *reinterpret_cast<f32x4*>(p.a.part_o + part * HD + 16 * db + 4 * g4) = acc[db];
      if (g4 == 0) *reinterpret_cast<float2*>(p.a.part_ml + 2 * part) = float2{st.m, l};
    };
    leave(end_col, l1, r1, o);
    leave(16 + end_col, l2, r2, o2);
    return;
  }
  auto store = [&](const Row& at, float l, const RowState& r, const f32x4 (&acc)[HD / 16]) {
    if (!at.valid) return;
    const int64_t tok = rq.tok_start + at.token;
    const float inv = 1.f / l;
    uint16_t* op = out_ptr(p.a, tok, at.head * HD + 4 * g4);
#pragma unroll
    for (int db = 0; db < HD / 16; db++) {
      u32x2 w;
      w[0] = pack_bf16x2(acc[db][0] * inv, acc[db][1] * inv);
      w[1] = pack_bf16x2(acc[db][2] * inv, acc[db][3] * inv);
      *reinterpret_cast<u32x2*>(op + (db >> 1) * step32 + (db & 1) * 16) = w;
    }
    if (TRACK && g4 == 0) p.lse[tok * p.a.nq + at.head] = r.m + log2f(l);
  };
  store(row_at(row0 + end_col), l1, r1, o);
  store(row_at(row0 + 16 + end_col), l2, r2, o2);
}

// Launches of decode splits alone run a kernel of their own: without the prefill
// tiles' registers and LDS, three waves fit a SIMD.
template <int HD, bool TRACK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void decode_attn_f8_kernel(
    AttnF8Params p) {
  __shared__ __attribute__((aligned(16))) char smem[(4 * 16 * (HD + 4) + 2 * 4 * 16) * 4];
  const AttnItem it = p.a.items[blockIdx.x];
  decode_item<HD, true, TRACK>(p, it, p.a.reqs[it.req], smem);
}

template <int HD, bool TRACK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void paged_attn_f8_kernel(
    AttnF8Params p) {
  __shared__ __attribute__((aligned(16))) char smem[smem_bytes<HD>()];
  const AttnItem it = p.a.items[blockIdx.x];
  const ReqDev rq = p.a.reqs[it.req];
  if (it.kind == 1)
    prefill_item<HD, TRACK>(p, it, rq, smem);
  else
    decode_item<HD, false, TRACK>(p, it, rq, smem);
}

struct SmallAttn {
  AttnF8Params p;
  InlineMeta meta;
};
template <int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void small_attn_f8_kernel(
    SmallAttn a) {
  __shared__ __attribute__((aligned(16))) char smem[smem_bytes<HD>()];
  AttnF8Params p = a.p;
  p.a.reqs = inline_meta(offsetof(SmallAttn, meta), p.a.reqs);
  p.a.pages = inline_meta(offsetof(SmallAttn, meta), p.a.pages);
  p.a.items = inline_meta(offsetof(SmallAttn, meta), p.a.items);
  const AttnItem it = p.a.items[blockIdx.x];
  const ReqDev rq = p.a.reqs[it.req];
  if (it.kind == 1)
    prefill_item<HD, false>(p, it, rq, smem);
  else
    decode_item<HD, true, false>(p, it, rq, smem);
}

// ---------------------------------------------------------------- attention weights
// Added with an atomic: requests of a batch may share the pages of a cached prefix,
// and then several workgroups add to one token.
__device__ __forceinline__ void add_weight(float* w, float x) { unsafeAtomicAdd(w, x); }

// Merges the splits of a prefill tile over its keys: HD / 4 threads a row, 8 (HD = 128) or
// 16 rows of one unit a workgroup.  Bound by memory (1024 rows of 32 heads in two splits,
// 34 MB of partials just written, beside the weights of 16 decodes: 10 us, 5 those alone).
template <int HD>
constexpr int kMergeRows = 4 * kMergeThreads / HD;
template <int HD>
__device__ __forceinline__ void merge_tile(const AttnF8Params& p, const TileMerge* tiles, int index) {
  constexpr int BLOCKS = kPrefillTileRows / kMergeRows<HD>;
  const int shift = p.pack_log2, units = p.a.nq >> shift;
  const TileMerge tm = tiles[index / BLOCKS / units];
  const ReqDev rq = p.a.reqs[tm.req];
  const int unit = index / BLOCKS % units;
  const int r = index % BLOCKS * kMergeRows<HD> + threadIdx.x / (HD / 4), d = 4 * (threadIdx.x % (HD / 4));
  const int row = tm.start + r;
  if (row >= rq.n_new << shift) return;
  const int64_t base = (int64_t)tm.part + unit * tm.n_split * kPrefillTileRows + r;
  float m = kNegBig, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < tm.n_split; s++) {
    const int64_t at = base + s * kPrefillTileRows;
    const float2 ml = *reinterpret_cast<const float2*>(p.a.part_ml + 2 * at);
    const f32x4 o = *reinterpret_cast<const f32x4*>(p.a.part_o + at * HD + d);
    const float mn = fmaxf(m, ml.x);
    const float a = exp2f(m - mn), w = exp2f(ml.x - mn);
    acc = acc * a + o * w;
    l = l * a + ml.y * w;
    m = mn;
  }
  const int64_t tok = rq.tok_start + (row >> shift);
  const int head = (unit << shift) + (row & ((1 << shift) - 1));
  const float inv = 1.f / l;
  u32x2 w;
  w[0] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  w[1] = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(out_ptr(p.a, tok, head * HD + d)) = w;
  if (p.weight && d == 0) p.lse[tok * p.a.nq + head] = m + log2f(l);
}

// What follows the attention in one launch: the accumulation of decodes' weights, the
// merge of decodes' key splits and that of prefill tiles'.  The first is
//   weight[slot][g] += sum over the q heads h of group g of exp2(score - lse[h]),
// the scores as the attention left them, lse from the splits' own maxima and sums
// (which the merge combines to the same) or, unsplit, as the attention left it.
// weights: four keys per thread, 256 apart, so that the adds of a wave are one run
// (four neighbouring keys per thread took 30 us for 64 requests of 300 to 8192 tokens
// of the 8B heads, 10 this way).
template <int HD>
__global__ __launch_bounds__(kMergeThreads) void finish_kernel(AttnF8Params p,
                                                               const WeightItem* items, int n_weights,
                                                               const MergeItem* merges, int n_merges,
                                                               const TileMerge* tiles) {
  __shared__ __attribute__((aligned(16))) float smem[merge_floats<HD>()];
  static_assert(kWeightDecodePages == 64 && kMergeThreads == 256, "four rounds of 256 keys");
  if ((int)blockIdx.x >= n_weights) {
    const int i = blockIdx.x - n_weights;
    if (i < n_merges) merge_splits<HD>(p.a, merges[i / p.a.nq], i % p.a.nq, smem);
    else merge_tile<HD>(p, tiles, i - n_merges);
    return;
  }
  const WeightItem it = items[blockIdx.x / p.a.nkv];
  const ReqDev rq = p.a.reqs[it.req];
  const int g = blockIdx.x % p.a.nkv, group = p.a.group;
  const int64_t len = score_row(rq.n_pages);
  const float* s = p.scores + p.score_base[it.req] + (int64_t)g * group * len;
  const int t = threadIdx.x, key0 = it.start * 16 + t;
  int key[4];  // (past the request: its last key, whose sum is not used)
  int64_t page[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    key[i] = min(key0 + 256 * i, rq.kv_len - 1);
    page[i] = p.a.pages[rq.page_start + (key[i] >> 4)];
  }
  float w[4] = {0.f, 0.f, 0.f, 0.f};
  for (int h0 = 0; h0 < group; h0 += 16) {  // 16 heads at a time, 16 threads each for lse
    const int h = g * group + h0 + (t >> 4);
    float m = kNegBig, l = 0.f;
    if (h0 + (t >> 4) < group) {
      if (rq.n_split == 1) {
        m = p.lse[(int64_t)rq.tok_start * p.a.nq + h];
        l = (t & 15) == 0 ? 1.f : 0.f;
      } else {
        const float2* ml = reinterpret_cast<const float2*>(p.a.part_ml) + it.part + (int64_t)h * rq.n_split;
        for (int k = t & 15; k < rq.n_split; k += 16) {
          const float2 x = ml[k];
          const float mn = fmaxf(m, x.x);
          l = l * exp2f(m - mn) + x.y * exp2f(x.x - mn);
          m = mn;
        }
      }
    }
    float M = m;
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) M = fmaxf(M, __shfl_xor(M, x));
    l *= exp2f(m - M);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) l += __shfl_xor(l, x);
    if ((t & 15) == 0) smem[t >> 4] = M + log2f(l);
    __syncthreads();
    const int heads = min(16, group - h0);
#pragma unroll 4
    for (int k = 0; k < heads; k++) {
      const float lse = smem[k];
#pragma unroll
      for (int i = 0; i < 4; i++) w[i] += fast_exp2(s[(h0 + k) * len + key[i]] - lse);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (key0 + 256 * i < rq.kv_len)
      add_weight(p.weight + (page[i] * p.a.nkv + g) * 16 + (key0 & 15), w[i]);
}

// The same for a prefill chunk, whose scores are computed again: a wave holds 64 keys
// of one KV head in registers, and the four waves of a workgroup, 256 keys, go through
// the group's query rows together, 32 rows of a head at a time through LDS, the next 32
// in flight meanwhile.  (Read from global memory by the lanes that need them the rows
// took longer than all the rest: they lie a power of two apart, in one L1 set and on
// few L2 channels.  1024 tokens over 4001, 8B heads: 112 us against 64.)  Where
// there are few keys the rows are split into parts (p.parts); each leaves its sums in
// the workspace, and a second launch adds them up in order.
//
// In LDS the 16-byte piece j of row r lies at j ^ row_swizzle(r), so that the 16 lanes
// it serves at a time hit distinct bank groups.
constexpr int kWeightRows = 32;
template <int HD>
__device__ __forceinline__ int row_swizzle(int r) {
  if constexpr (HD == 128) return r & 15;
  else return ((r >> 1) & 5) | ((r >> 2) & 2);
}
template <int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void weight_prefill_kernel(
    AttnF8Params p, const WeightItem* items) {
  __shared__ u32x4 s_q[2][kWeightRows * HD / 8];
  __shared__ float s_lse[2][kWeightRows];
  const int g = blockIdx.x % p.a.nkv, tile = blockIdx.x / p.a.nkv / p.parts;
  const int part = blockIdx.x / p.a.nkv % p.parts;
  const WeightItem it = items[tile];
  const ReqDev rq = p.a.reqs[it.req];
  const int group = p.a.group;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g4 = lane >> 4;
  const int page0 = it.start + 4 * wave, page = page0 + g4;  // the wave's pages, this lane's
  bf16x8 kf[4][HD / 32];
  {
    const int id = p.a.pages[rq.page_start + min(page0 + (col >> 2), rq.n_pages - 1)];
    const int64_t kp = (int64_t)id * p.a.nkv + g;
    const uint8_t* k = p.k8 + kp * (16 * HD) + (col & 3) * 64 + 16 * g4;
    const float ks = p.k_scale[kp];
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int h = 0; h < HD / 64; h++) {
        const u32x4 c = *reinterpret_cast<const u32x4*>(k + h * 1024 + b * 256);
        kf[b][2 * h] = widen(c[0], c[1], ks);
        kf[b][2 * h + 1] = widen(c[2], c[3], ks);
      }
  }
  float acc[4][4] = {};
  // Row blocks from the first that sees one of the 256 keys on, this part's share of them.
  const int first_key = it.start * 16, blocks = (rq.n_new + kWeightRows - 1) / kWeightRows;
  const int blk0 = max(0, first_key - rq.ctx_len) / kWeightRows;
  const int share = (blocks - blk0 + p.parts - 1) / p.parts;
  const int begin = blk0 + part * share, end = min(begin + share, blocks);

  // this thread's pieces of a block of rows, and a row's log-sum (infinite past the last
  // row, which then adds 0)
  constexpr int PIECES = HD / 8, NP = kWeightRows * PIECES / 256;
  u32x4 piece[NP];
  float row_lse = 0.f;
  auto fetch = [&](int blk, int head) {
    const int h = g * group + head;
#pragma unroll
    for (int i = 0; i < NP; i++) {
      const int u = threadIdx.x + 256 * i;
      const int64_t tok = rq.tok_start + min(kWeightRows * blk + u / PIECES, rq.n_new - 1);
      piece[i] = *reinterpret_cast<const u32x4*>(p.a.q + tok * p.a.q_tok_stride + (int64_t)h * HD +
                                                 8 * (u % PIECES));
    }
    if (threadIdx.x < kWeightRows) {
      const int row = kWeightRows * blk + threadIdx.x;
      row_lse = row < rq.n_new ? p.lse[(int64_t)(rq.tok_start + row) * p.a.nq + h] : __builtin_inff();
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NP; i++) {
      const int u = threadIdx.x + 256 * i, r = u / PIECES;
      s_q[buf][r * PIECES + ((u % PIECES) ^ row_swizzle<HD>(r))] = piece[i];
    }
    if (threadIdx.x < kWeightRows) s_lse[buf][threadIdx.x] = row_lse;
  };
  auto add = [&](auto mask, int buf, int row0, int sub) {  // 16 rows of the block
    const int r = 16 * sub + col;
    bf16x8 q[HD / 32];
#pragma unroll
    for (int e = 0; e < HD / 32; e++)  // dims 64 (e / 2) + 16 g4 + 8 (e % 2) .. + 7
      q[e] = as_bf16x8(s_q[buf][r * PIECES + ((8 * (e >> 1) + 2 * g4 + (e & 1)) ^ row_swizzle<HD>(r))]);
    const float lse = s_lse[buf][r];
    f32x4 s[4];
#pragma unroll
    for (int b = 0; b < 4; b++) s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < HD / 32; e++)
#pragma unroll
      for (int b = 0; b < 4; b++) s[b] = mfma16(kf[b][e], q[e], s[b]);
    const int last = rq.ctx_len + row0 + r - page * 16;  // the page's last token that counts
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float w = fast_exp2(fmaf(s[b][i], p.a.scale_log2, -lse));
        acc[b][i] += !decltype(mask)::value || 4 * b + i <= last ? w : 0.f;
      }
  };
  if (begin < end) {
    fetch(begin, 0);
    put(0);
    __syncthreads();
    int blk = begin, head = 0;
    for (int buf = 0; blk < end; buf ^= 1) {
      int nblk = blk, nhead = head + 1;
      if (nhead == group) {
        nhead = 0;
        nblk++;
      }
      if (nblk < end) fetch(nblk, nhead);
      const int row0 = kWeightRows * blk;
#pragma unroll
      for (int sub = 0; sub < kWeightRows / 16; sub++) {
        // (how far the first row's position is past the wave's first key)
        const int past = rq.ctx_len + row0 + 16 * sub - page0 * 16;
        if (past >= 63) add(std::integral_constant<bool, false>{}, buf, row0, sub);
        else if (past > -16) add(std::integral_constant<bool, true>{}, buf, row0, sub);
      }
      if (nblk < end) put(buf ^ 1);
      __syncthreads();
      blk = nblk;
      head = nhead;
    }
  }
  // the sums over the 16 rows of a block: lane 16 g4 + col keeps token col of page g4
  float w = 0.f;
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
      for (int m = 1; m < 16; m <<= 1) acc[b][i] += __shfl_xor(acc[b][i], m);
      if (col == 4 * b + i) w = acc[b][i];
    }
  const int key = page * 16 + col;
  if (p.parts > 1)
    p.part_w[(int64_t)blockIdx.x * 256 + threadIdx.x] = w;
  else if (key < rq.kv_len)
    add_weight(p.weight + ((int64_t)p.a.pages[rq.page_start + page] * p.a.nkv + g) * 16 + col, w);
}

// Adds the parts' sums of 256 keys of one KV head.
__global__ __launch_bounds__(256) void weight_parts_kernel(AttnF8Params p, const WeightItem* items) {
  const int g = blockIdx.x % p.a.nkv, tile = blockIdx.x / p.a.nkv;
  const WeightItem it = items[tile];
  const ReqDev rq = p.a.reqs[it.req];
  const int key = it.start * 16 + (int)threadIdx.x;
  if (key >= rq.kv_len) return;
  const float* w = p.part_w + ((int64_t)tile * p.parts * p.a.nkv + g) * 256 + threadIdx.x;
  float sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < p.parts; i++) sum += w[(int64_t)i * p.a.nkv * 256];
  const int64_t id = p.a.pages[rq.page_start + (key >> 4)];
  add_weight(p.weight + (id * p.a.nkv + g) * 16 + (key & 15), sum);
}

template <int HD>
hipError_t launch(const AttnF8Params& p, int n_items, const MergeItem* merges, int n_merges,
                  const TileMerge* tiles, int n_tiles, const WeightItem* dec, int n_dec,
                  const WeightItem* pre, int n_pre, hipStream_t stream) {
  if (n_items > 0) {
    if (p.a.decode_only && p.weight)
      decode_attn_f8_kernel<HD, true><<<n_items, 256, 0, stream>>>(p);
    else if (p.a.decode_only)
      decode_attn_f8_kernel<HD, false><<<n_items, 256, 0, stream>>>(p);
    else if (p.weight)
      paged_attn_f8_kernel<HD, true><<<n_items, 256, 0, stream>>>(p);
    else
      paged_attn_f8_kernel<HD, false><<<n_items, 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipError_t e = hipSuccess;
  const int weights = n_dec * p.a.nkv, rows = n_merges * p.a.nq;
  const int blocks = kPrefillTileRows / kMergeRows<HD> * (p.a.nq >> p.pack_log2);
  if (const int n = weights + rows + n_tiles * blocks; n > 0) {
    finish_kernel<HD><<<n, kMergeThreads, 0, stream>>>(p, dec, weights, merges, rows, tiles);
    e = hipGetLastError();
  }
  if (e == hipSuccess && n_pre > 0) {
    weight_prefill_kernel<HD><<<n_pre * p.parts * p.a.nkv, 256, 0, stream>>>(p, pre);
    if ((e = hipGetLastError()) != hipSuccess || p.parts == 1) return e;
    weight_parts_kernel<<<n_pre * p.a.nkv, 256, 0, stream>>>(p, pre);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_small_attn_f8(const AttnF8Params& p, const InlineMeta& meta, int n_items,
                                int head_dim, hipStream_t stream) {
  if (n_items == 0) return hipSuccess;
  const SmallAttn a{p, meta};
  if (head_dim == 128)
    small_attn_f8_kernel<128><<<n_items, 256, 0, stream>>>(a);
  else
    small_attn_f8_kernel<64><<<n_items, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_attn_f8(const AttnF8Params& p, int n_items, const MergeItem* merges,
                                int n_merges, const TileMerge* tiles, int n_tiles,
                                const WeightItem* dec, int n_dec, const WeightItem* pre, int n_pre,
                                int head_dim, hipStream_t stream) {
  const auto call = head_dim == 128 ? launch<128> : launch<64>;
  return call(p, n_items, merges, n_merges, tiles, n_tiles, dec, n_dec, pre, n_pre, stream);
}

}  // namespace mx
