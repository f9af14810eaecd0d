// attention_bf16.h -- what the attention kernels over the bf16 cache share: a 32-key
// step's loads, score and value products, and the copies of a prefill tile's keys.
#pragma once

#include "attention_tile.h"

namespace mx {

namespace {

template <int HD>
struct Chunk {
  u32x4 k[2][HD / 32];  // keys: 16 B per lane per (score block, d-step)
  u32x4 v[HD / 16];     // values (transposed pages): 16 B per lane per d-block
};

// Key order inside a 32-key step (two pages).  Score block b, row m holds key
//   kappa_b(m) = 8 * (m / 4) + 4 * b + m % 4,
// so that lane group g (rows 4g .. 4g+3 of both blocks) ends up with the eight
// consecutive keys 8g .. 8g+7, all in page g / 2.  Those eight keys are then
// one 16-byte run of a transposed value page, and they are exactly the k
// indices the second product expects from this lane group.
// Non-temporal loads (streamed past the caches' retention): every key and
// value of a decode split is read once.  A value load reads whole 128-byte
// lines (16 dim rows x 32 bytes of a page, contiguous), so its values are
// always loaded non-temporally.  Keys are non-temporal (NT) only in launches
// of decode splits alone.  With token-major key pages a key load read half
// lines, and beside prefill tiles (whose copies keep the L2 busy) non-temporal
// keys made the launch slower (70B at P = 4096: 2.19 ms against 1.88 ms); with
// the blocked key pages every key load reads whole lines, and non-temporal
// keys in mixed launches measured no better than ordinary ones.  Measured:
// decode-only attention 3-11% faster on the four layer shapes (7B 70.0 ->
// 78.1% of the HBM peak, 13B 70.6 -> 75.8%, Llama-3-8B 70.8 -> 78.8%, 70B
// 78.2 -> 80.3%); non-temporal values in mixed launches 1-3.5% faster (70B,
// P = 1024 .. 8192).
template <int HD, bool NT>
__device__ __forceinline__ u32x4 stream_load(const uint16_t* ptr) {
  const u32x4* q = reinterpret_cast<const u32x4*>(ptr);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  else return *q;
}

template <int HD, bool NT>
__device__ __forceinline__ void load_chunk(Chunk<HD>& c, const AttnParams& p, int kvh, int pid0,
                                           int pid1, int safe, int col, int g4) {
  // A page id of -1 (past the split's end) reads the request's first page
  // instead: those keys and values are masked out by select in
  // process_chunk, and every load stays unconditional, which keeps the
  // count of loads in flight the same on every path.
  // keys: lane row m = col; its key kappa_b(col) lives in page col / 8.  A key
  // page is blocked by 32 dims ([d / 32][16 slots][32]), so the four
  // consecutive slots that rows 4i .. 4i + 3 read of a 32-dim block in one
  // load are one contiguous 256-byte run: every load moves whole 128-byte
  // lines.
  {
    const int page0 = (col < 8) ? pid0 : pid1;
    const int page = page0 >= 0 ? page0 : safe;
    const int slot0 = 8 * ((col >> 2) & 1) + (col & 3);
    const uint16_t* kb_ptr = p.k_pool + ((int64_t)page * p.nkv + kvh) * (int64_t)(16 * HD);
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int ds = 0; ds < HD / 32; ds++)
        c.k[b][ds] = stream_load<HD, NT>(kb_ptr + ds * 512 + (slot0 + 4 * b) * 32 + 8 * g4);
  }
  // values: lane group g reads keys 8 (g % 2) .. +7 of page g / 2 at d = 16 db + col
  {
    const int page0 = (g4 < 2) ? pid0 : pid1;
    const int page = page0 >= 0 ? page0 : safe;
    const uint16_t* vb_ptr = p.v_pool + ((int64_t)page * p.nkv + kvh) * (int64_t)(16 * HD) + 8 * (g4 & 1);
#pragma unroll
    for (int db = 0; db < HD / 16; db++)
      c.v[db] = stream_load<HD, true>(vb_ptr + (db * 16 + col) * 16);
  }
}

// Score block b of S^T = K Q^T (16 keys x 16 rows).
template <int HD>
__device__ __forceinline__ f32x4 score_block(const u32x4 (&kf)[HD / 32], const bf16x8 (&qf)[HD / 32]) {
  f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ds = 0; ds < HD / 32; ds++) s = mfma16(as_bf16x8(kf[ds]), qf[ds], s);
  return s;
}

// The step's probabilities of this lane's keys, exp2(score * scale - m), as
// the value product's B operand (k index i' = 4 b + i <-> key j0 + i'), and
// their sum into the lane's share of the row's sum: two at a time with the
// bf16 dot instruction, from the same rounded values the value product uses.
__device__ __forceinline__ bf16x8 probs(const float (&sv)[2][4], RowState& r, float scale_log2) {
  float pv[2][4];
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int i = 0; i < 4; i++) pv[b][i] = fast_exp2(fmaf(sv[b][i], scale_log2, -r.m));
  // Four separate words, put together only for the return: with the words
  // taken out of a four-word vector, this compiler's dot instructions all
  // read its first word.
  const uint32_t w0 = pack_bf16x2(pv[0][0], pv[0][1]);
  const uint32_t w1 = pack_bf16x2(pv[0][2], pv[0][3]);
  const uint32_t w2 = pack_bf16x2(pv[1][0], pv[1][1]);
  const uint32_t w3 = pack_bf16x2(pv[1][2], pv[1][3]);
  const mx_bf16x2 ones = __builtin_bit_cast(mx_bf16x2, 0x3F803F80u);
  r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w0), ones, r.l, false);
  r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w1), ones, r.l, false);
  r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w2), ones, r.l, false);
  r.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, w3), ones, r.l, false);
  return as_bf16x8(u32x4{w0, w1, w2, w3});
}

// O^T += V^T P^T over the output blocks DB0 .. DB0 + NDB - 1 (16 head dims
// each), V^T as the A operand.
template <int HD, int DB0, int NDB, bool MASK>
__device__ __forceinline__ void values_part(const u32x4 (&vf)[NDB], f32x4 (&o)[HD / 16], bf16x8 pb,
                                            const uint32_t (&keep)[4]) {
#pragma unroll
  for (int e = 0; e < NDB; e++) {
    u32x4 va = vf[e];
    if constexpr (MASK) {
#pragma unroll
      for (int h = 0; h < 4; h++) va[h] &= keep[h];
    }
    o[DB0 + e] = mfma16(as_bf16x8(va), pb, o[DB0 + e]);
  }
}

// Prefill tiles share every 32-key chunk through LDS.  The four waves copy it
// there with the DMA path (global_load_lds, 16 bytes per lane), a quarter each
// (waves 0 and 1 the keys of the chunk's two pages, waves 2 and 3 their
// values), and every wave reads its matrix-core fragments from there.  Keys
// are stored [32][HD] with the 16-byte chunk c of key row j at c ^ ksw(j);
// values page by page, [2 pages][HD][2 halves of 8 keys], unswizzled.  Both make
// the 16 lanes that the LDS serves at a time ({0-3, 12-15, 20-23, 24-27} and so
// on, not 16 consecutive ones) hit distinct bank groups: 4.2 clocks per read.
// (Value halves swapped for odd groups of 8 dim rows, which is conflict-free for
// 16 consecutive lanes, took 8.0.)  A DMA
// instruction writes 1 KB of LDS in lane order, so each lane fetches the 16
// bytes that belong at its position: a permutation within the page's rows
// (and, for keys, within its 32-dim blocks), which keeps every copy a run of
// whole 128-byte lines.  A wave's copies of a chunk all read one page (even waves
// the first, odd waves the second), so its address is scalar arithmetic, once per
// chunk.
template <int HD>
__device__ __forceinline__ int ksw(int key) {
  if constexpr (HD == 128) return (key & 3) | ((key >> 3) << 2);
  else return ((key >> 1) & 1) | ((key >> 3) << 1);
}
template <int HD>
struct SharedChunk {
  static constexpr int KBYTES = 32 * HD * 2;
  static constexpr int BYTES = 2 * KBYTES;  // keys + values
  static constexpr int SLOTS = 4;           // chunks kt .. kt + 3: copies run three ahead
  static constexpr int NLD = BYTES / 4096;  // 1 KB copies per wave per chunk
};
template <int HD>
constexpr int smem_bytes() {
  constexpr int ring = SharedChunk<HD>::SLOTS * SharedChunk<HD>::BYTES;
  constexpr int combine = (4 * 16 * (HD + 4) + 2 * 4 * 16) * 4;
  return ring > combine ? ring : combine;
}

}  // namespace

}  // namespace mx
