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
// Keys are consumed four pages (64 keys) at a time.  Score block b, row m is the key
//   kappa_b(m) = token 4 b + m % 4 of page m / 4,
// so that lane group g (rows 4 g .. 4 g + 3 of the four blocks) ends up with the 16
// tokens of page g: one scale per lane for its values, and the tokens of a value
// row of that page are one 16-byte run, in the order the second product takes them.
#include <type_traits>

#include "attention_tile.h"

namespace mx {

namespace {

template <int HD>
struct Chunk8 {
  u32x4 k[4][HD / 64];  // key codes: 16 dims of one key per lane per (score block, 64 dims)
  u32x4 v[HD / 16];     // value codes: the 16 tokens of a page per lane per 16 dims
  float ks, vs;         // scales of the lane's key page and of its value page
};

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

// The keys of the step that starts at page pi: page ids of this lane's key and
// value pages (past the range: its last page, whose keys are masked there).
struct PageIds {
  int k, v;
};
__device__ __forceinline__ PageIds page_ids(const int32_t* ptab, int pi, int page_end, int col,
                                            int g4) {
  return PageIds{ptab[min(pi + (col >> 2), page_end - 1)], ptab[min(pi + g4, page_end - 1)]};
}

template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint8_t* ptr) {
  const u32x4* q = reinterpret_cast<const u32x4*>(ptr);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  else return *q;
}

template <int HD, bool NT>
__device__ __forceinline__ void load_chunk(Chunk8<HD>& c, const AttnF8Params& p, int kvh,
                                           const PageIds& id, int col, int g4) {
  const int64_t kp = (int64_t)id.k * p.a.nkv + kvh, vp = (int64_t)id.v * p.a.nkv + kvh;
  const uint8_t* k = p.k8 + kp * (16 * HD) + (col & 3) * 64 + 16 * g4;
  const uint8_t* v = p.v8 + vp * (16 * HD) + col * 16;
  c.ks = p.k_scale[kp];
  c.vs = p.v_scale[vp];
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int h = 0; h < HD / 64; h++) c.k[b][h] = load16<NT>(k + h * 1024 + b * 256);
#pragma unroll
  for (int db = 0; db < HD / 16; db++) c.v[db] = load16<true>(v + db * 256);
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

// This lane's 16 raw scores of the step (keys past the range or after the row's
// position masked to kNegBig by select) and their max.
template <bool MASK>
__device__ __forceinline__ float masked_scores(const f32x4 (&s)[4], float (&sv)[4][4], int page,
                                               int page_end, int row_pos) {
  float mx = kNegBig;
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      sv[b][i] = (!MASK || (page < page_end && page * 16 + 4 * b + i <= row_pos)) ? s[b][i] : kNegBig;
      mx = fmaxf(mx, sv[b][i]);
    }
  return mx;
}

// The step's probabilities of this lane's keys, exp2(score * scale - m), as the
// B operands of the value products (product i: tokens 8 i .. 8 i + 7 of the lane's
// page), and their sum into the lane's share of the row's sum: from the rounded
// values that the products use, or (EXACT) from the values before that rounding,
// which the accumulated weights need: theirs is an fp32 result, and the rounded
// sum of a row is off by up to 2^-9.
template <bool EXACT>
__device__ __forceinline__ void probs(const float (&sv)[4][4], RowState& r, float scale_log2,
                                      bf16x8 (&pb)[2]) {
  const mx_bf16x2 ones = __builtin_bit_cast(mx_bf16x2, 0x3F803F80u);
#pragma unroll
  for (int h = 0; h < 2; h++) {
    float pv[2][4];
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        pv[b][i] = fast_exp2(fmaf(sv[2 * h + b][i], scale_log2, -r.m));
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
    pb[h] = as_bf16x8(u32x4{w0, w1, w2, w3});
  }
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
template <int HD, int DB0, int NDB, bool MASK>
__device__ __forceinline__ void values_part(const u32x4 (&vf)[NDB], float vs, f32x4 (&o)[HD / 16],
                                            const bf16x8 (&pb)[2], const uint32_t (&keep)[4]) {
#pragma unroll
  for (int e = 0; e < NDB; e++) {
    u32x4 v = vf[e];
    if constexpr (MASK) {
#pragma unroll
      for (int w = 0; w < 4; w++) v[w] &= keep[w];
    }
    o[DB0 + e] = mfma16(widen(v[0], v[1], vs), pb[0], o[DB0 + e]);
    o[DB0 + e] = mfma16(widen(v[2], v[3], vs), pb[1], o[DB0 + e]);
  }
}

// What a wave's 16 query rows scan: pages first, first + step .. of those below
// page_end, 64 keys each (four pages), up to the row's own position.
struct Scan {
  int first, step, page_end, row_pos, first_row_pos, kv_len;
};

// One 64-key step of the online softmax for this lane's query row.  scores: where
// to leave the lane's 16 scores in log2 units, or null.
template <int HD, bool MASK, bool TRACK>
__device__ __forceinline__ void process_chunk(const Chunk8<HD>& c, const bf16x8 (&qf)[HD / 32],
                                              f32x4 (&o)[HD / 16], RowState& r, int pi,
                                              const Scan& sc, float scale_log2, float inv_scale,
                                              int g4, float* scores) {
  f32x4 s[4];
#pragma unroll
  for (int b = 0; b < 4; b++) s[b] = score_block<HD>(c.k[b], c.ks, qf);
  float sv[4][4];
  const int page = pi + g4;
  const float mx = masked_scores<MASK>(s, sv, page, sc.page_end, sc.row_pos);
  if constexpr (TRACK) {
    if (scores && (!MASK || page < sc.page_end)) {
#pragma unroll
      for (int b = 0; b < 4; b++)
        *reinterpret_cast<f32x4*>(scores + page * 16 + 4 * b) =
            f32x4{sv[b][0], sv[b][1], sv[b][2], sv[b][3]} * scale_log2;
    }
  }
  if (__any(mx > r.thr)) raise_max(r, mx, scale_log2, inv_scale, o);
  bf16x8 pb[2];
  probs<TRACK>(sv, r, scale_log2, pb);
  uint32_t keep[4];
  value_keep(page, sc.page_end, sc.kv_len, keep);
  values_part<HD, 0, HD / 16, MASK>(c.v, c.vs, o, pb, keep);
}

// The scan from global memory: two chunk buffers used in turn, the next chunk's
// loads in flight while the current one is processed, page ids fetched one chunk
// ahead of their loads.  Unrolled by two so that no buffer is ever copied.
template <int HD, bool NT, bool TRACK>
__device__ __forceinline__ void scan_rows(const AttnF8Params& p, const int32_t* ptab, int kvh,
                                          const Scan& sc, const bf16x8 (&qf)[HD / 32],
                                          f32x4 (&o)[HD / 16], RowState& r, int col, int g4,
                                          float* scores) {
  const float scale = p.a.scale_log2, inv_scale = 1.f / scale;
  auto ids = [&](int pi) { return page_ids(ptab, pi, sc.page_end, col, g4); };
  auto proc = [&](const Chunk8<HD>& c, int pi) {
    // all 64 keys count for every row of the wave: no mask is needed
    if (pi + 3 < sc.page_end && pi * 16 + 63 <= sc.first_row_pos)
      process_chunk<HD, false, TRACK>(c, qf, o, r, pi, sc, scale, inv_scale, g4, scores);
    else
      process_chunk<HD, true, TRACK>(c, qf, o, r, pi, sc, scale, inv_scale, g4, scores);
  };
  int pi = sc.first;
  if (pi >= sc.page_end) return;
  Chunk8<HD> ca, cb;
  PageIds n = ids(pi + sc.step);
  load_chunk<HD, NT>(ca, p, kvh, ids(pi), col, g4);
  while (true) {
    int pn = pi + sc.step;
    if (pn >= sc.page_end) {
      proc(ca, pi);
      break;
    }
    PageIds nn = ids(pn + sc.step);
    load_chunk<HD, NT>(cb, p, kvh, n, col, g4);
    proc(ca, pi);
    pi = pn;
    n = nn;
    pn = pi + sc.step;
    if (pn >= sc.page_end) {
      proc(cb, pi);
      break;
    }
    nn = ids(pn + sc.step);
    load_chunk<HD, NT>(ca, p, kvh, n, col, g4);
    proc(cb, pi);
    pi = pn;
    n = nn;
  }
}

// Decode item: the q heads it.head .. it.head + nrows - 1 (one per lane row) of the
// request's single token, over pages it.start .. of its table; the four waves
// stride over the split's 64-key chunks and combine through LDS.
template <int HD, bool NT, bool TRACK>
__device__ __forceinline__ void decode_item(const AttnF8Params& p, const AttnItem& it,
                                            const ReqDev& rq, char* smem) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
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
  Scan sc;
  sc.first = it.start + 4 * wave;
  sc.step = 16;
  sc.page_end = min(it.start + p.a.split_pages, rq.n_pages);
  sc.row_pos = sc.first_row_pos = rq.kv_len - 1;
  sc.kv_len = rq.kv_len;
  float* scores = nullptr;
  if constexpr (TRACK) {
    if (row_valid) scores = p.scores + p.score_base[it.req] + (int64_t)qhead * 16 * rq.n_pages;
  }
  scan_rows<HD, NT, TRACK>(p, p.a.pages + rq.page_start, it.head / p.a.group, sc, qf, o, r, col, g4,
                           scores);

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
    if (TRACK && (threadIdx.x & 15) == 0) p.a.lse[qtok * p.a.nq + h] = M + log2f(L);
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

// Prefill item: one q head, rows it.start .. it.start + 127 of the chunk, two
// blocks of 16 rows per wave.
template <int HD, bool TRACK>
__device__ __forceinline__ void prefill_item(const AttnF8Params& p, const AttnItem& it,
                                             const ReqDev& rq) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int col = lane & 15;  // query row of this lane within the block
  const int g4 = lane >> 4;
  for (int blk = 0; blk < 2; blk++) {
    const int row0 = it.start + 32 * wave + 16 * blk;
    if (row0 >= rq.n_new) return;
    const int row = min(row0 + col, rq.n_new - 1);
    const int64_t qtok = rq.tok_start + row;
    RowState r = row_start();
    f32x4 o[HD / 16];
#pragma unroll
    for (int db = 0; db < HD / 16; db++) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 qf[HD / 32];
    load_q<HD>(p, qtok, it.head, true, g4, qf);
    Scan sc;
    sc.first = 0;
    sc.step = 4;
    sc.row_pos = rq.ctx_len + row;
    sc.first_row_pos = rq.ctx_len + row0;
    sc.page_end = (rq.ctx_len + min(row0 + 15, rq.n_new - 1)) / 16 + 1;
    sc.kv_len = rq.kv_len;
    scan_rows<HD, false, TRACK>(p, p.a.pages + rq.page_start, it.head / p.a.group, sc, qf, o, r,
                                col, g4, nullptr);
    const float l = lane_groups_sum(r.l);
    if (row0 + col >= rq.n_new) continue;
    const float inv = 1.f / l;
    const int64_t step32 = p.a.out_tiled ? 512 : 32;
    uint16_t* op = out_ptr(p.a, qtok, it.head * HD + 4 * g4);
#pragma unroll
    for (int db = 0; db < HD / 16; db++) {
      u32x2 w;
      w[0] = pack_bf16x2(o[db][0] * inv, o[db][1] * inv);
      w[1] = pack_bf16x2(o[db][2] * inv, o[db][3] * inv);
      *reinterpret_cast<u32x2*>(op + (db >> 1) * step32 + (db & 1) * 16) = w;
    }
    if (TRACK && g4 == 0) p.a.lse[qtok * p.a.nq + it.head] = r.m + log2f(l);
  }
}

template <int HD, bool TRACK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void paged_attn_f8_kernel(
    AttnF8Params p) {
  __shared__ __attribute__((aligned(16))) char smem[(4 * 16 * (HD + 4) + 2 * 4 * 16) * 4];
  const AttnItem it = p.a.items[blockIdx.x];
  const ReqDev rq = p.a.reqs[it.req];
  if (it.kind == 1)
    prefill_item<HD, TRACK>(p, it, rq);
  else if (p.a.decode_only)
    decode_item<HD, true, TRACK>(p, it, rq, smem);
  else
    decode_item<HD, false, TRACK>(p, it, rq, smem);
}

// ---------------------------------------------------------------- attention weights
// Added with an atomic: requests of a batch may share the pages of a cached prefix,
// and then several workgroups add to one token.
__device__ __forceinline__ void add_weight(float* w, float x) { unsafeAtomicAdd(w, x); }

// weight[slot][g] += sum over the q heads h of group g of exp2(score - lse[h]), the
// scores as the attention left them: one thread per four keys.
template <int HD>
__global__ __launch_bounds__(256) void weight_decode_kernel(AttnF8Params p,
                                                            const WeightItem* items) {
  const WeightItem it = items[blockIdx.x];
  const ReqDev rq = p.a.reqs[it.req];
  const int g = blockIdx.y, group = p.a.group;
  const int key = it.start * 16 + 4 * threadIdx.x;
  if (key >= rq.kv_len) return;
  const int64_t len = 16 * (int64_t)rq.n_pages;
  const float* s = p.scores + p.score_base[it.req] + (int64_t)g * group * len + key;
  const float* lse = p.a.lse + (int64_t)rq.tok_start * p.a.nq + g * group;
  f32x4 w = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int h = 0; h < group; h++) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(s + h * len);
    const float l = lse[h];
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] += fast_exp2(x[i] - l);
  }
  const int64_t page = p.a.pages[rq.page_start + (key >> 4)];
  float* out = p.weight + (page * p.a.nkv + g) * 16 + (key & 15);
  for (int i = 0; i < 4; i++)
    if (key + i < rq.kv_len) add_weight(out + i, w[i]);
}

// The same for a prefill chunk, whose scores are computed again: a workgroup holds
// 64 keys of one KV head, its four waves take the 16-row blocks of the group's query
// rows in turn, and their sums meet in LDS.
template <int HD>
__global__ __launch_bounds__(256) void weight_prefill_kernel(AttnF8Params p,
                                                             const WeightItem* items) {
  __shared__ float s_w[4][64];
  const WeightItem it = items[blockIdx.x];
  const ReqDev rq = p.a.reqs[it.req];
  const int g = blockIdx.y, group = p.a.group;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g4 = lane >> 4;
  const int page = it.start + g4;  // this lane's page
  bf16x8 kf[4][HD / 32];
  {
    const int id = p.a.pages[rq.page_start + min(it.start + (col >> 2), rq.n_pages - 1)];
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
  // rows before the first key see none of these keys
  const int blk0 = max(0, it.start * 16 - rq.ctx_len) / 16, blks = (rq.n_new + 15) / 16 - blk0;
  for (int t = wave; t < blks * group; t += 4) {
    const int row0 = 16 * (blk0 + t / group), head = g * group + t % group;
    const int row = row0 + col;
    const bool valid = row < rq.n_new;
    const int64_t tok = rq.tok_start + (valid ? row : rq.n_new - 1);
    bf16x8 qf[HD / 32];
    load_q<HD>(p, tok, head, true, g4, qf);
    const float lse = p.a.lse[tok * p.a.nq + head];
    const int row_pos = valid ? rq.ctx_len + row : -1;
#pragma unroll
    for (int b = 0; b < 4; b++) {
      f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < HD / 32; e++) s = mfma16(kf[b][e], qf[e], s);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float w = fast_exp2(fmaf(s[i], p.a.scale_log2, -lse));
        acc[b][i] += page * 16 + 4 * b + i <= row_pos ? w : 0.f;
      }
    }
  }
#pragma unroll
  for (int b = 0; b < 4; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
      for (int m = 1; m < 16; m <<= 1) acc[b][i] += __shfl_xor(acc[b][i], m);
      if (col == 4 * b + i) s_w[wave][lane] = acc[b][i];
    }
  __syncthreads();
  const int key = it.start * 16 + (int)threadIdx.x;
  if (threadIdx.x >= 64 || key >= rq.kv_len) return;
  const float w = (s_w[0][threadIdx.x] + s_w[1][threadIdx.x]) + (s_w[2][threadIdx.x] + s_w[3][threadIdx.x]);
  const int64_t id = p.a.pages[rq.page_start + (key >> 4)];
  add_weight(p.weight + (id * p.a.nkv + g) * 16 + (key & 15), w);
}

template <int HD>
hipError_t launch(const AttnF8Params& p, int n_items, const MergeItem* merges, int n_merges,
                  const WeightItem* dec, int n_dec, const WeightItem* pre, int n_pre,
                  hipStream_t stream) {
  if (n_items > 0) {
    if (p.weight)
      paged_attn_f8_kernel<HD, true><<<n_items, 256, 0, stream>>>(p);
    else
      paged_attn_f8_kernel<HD, false><<<n_items, 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipError_t e = launch_attn_merge(p.a, merges, n_merges, HD, stream);
  if (e != hipSuccess || !p.weight) return e;
  if (n_dec > 0) {
    weight_decode_kernel<HD><<<dim3(n_dec, p.a.nkv), 256, 0, stream>>>(p, dec);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (n_pre > 0) {
    weight_prefill_kernel<HD><<<dim3(n_pre, p.a.nkv), 256, 0, stream>>>(p, pre);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_paged_attn_f8(const AttnF8Params& p, int n_items, const MergeItem* merges,
                                int n_merges, const WeightItem* dec, int n_dec,
                                const WeightItem* pre, int n_pre, int head_dim,
                                hipStream_t stream) {
  return head_dim == 128
             ? launch<128>(p, n_items, merges, n_merges, dec, n_dec, pre, n_pre, stream)
             : launch<64>(p, n_items, merges, n_merges, dec, n_dec, pre, n_pre, stream);
}

}  // namespace mx
