// attention_tile.h -- what the attention kernels share: the output's address, the
// online softmax of a query row held by four lanes, runs of LDS fragment reads, the
// merge of key splits.
#pragma once

#include "mx_device.h"
#include "mx_kernels.h"

namespace mx {

namespace {

constexpr float kNegBig = -1.0e30f;

// Element (token t, column c = head * HD + dim) of the attention output:
// [T][nq][HD] row-major, or the projection-input tile layout when out_tiled.
__device__ __forceinline__ uint16_t* out_ptr(const AttnParams& p, int64_t t, int64_t c) {
  return p.out + (p.out_tiled ? tile_index(t, c, p.out_tok_stride) : t * p.out_tok_stride + c);
}

// Online-softmax state of this lane's query row.  m is the running max of the
// scaled scores (log2 units) that every probability of the row refers to, thr
// the raw score above which m has to be raised (m + kLazyMax, unscaled), and
// l this lane's share of the row's sum: the probabilities of the lane's own
// keys only.  The four lanes of a row share m and every rescale, so the row's
// sum is the sum of their shares, taken once at the end.
struct RowState {
  float m, thr, l;
};
__device__ __forceinline__ RowState row_start() { return RowState{kNegBig, kNegBig, 0.f}; }

// A row's running max m (log2 units) is raised only when a score exceeds it by
// more than this: the probabilities exp2(x - m) then stay below 2^8, which bf16
// and fp32 hold at full relative precision, and the output is rescaled only on
// the steps where some row of the wave raised its max (rarely, past the first
// keys).  Output and sum always refer to the same m, so the normalised result
// is the softmax itself.
constexpr float kLazyMax = 8.0f;

// Max and sum of a query row's values over its four lane groups (lanes l,
// l ^ 16, l ^ 32, l ^ 48).  v_permlane16_swap and v_permlane32_swap with both
// operands equal to x leave, in every lane, the even-row (lower-half) value in
// the first result and the odd-row (upper-half) value in the second: the lane's
// own value and its partner's, in the same order in both lanes of a pair.  So
// each step is one VALU swap and one VALU op, with no LDS permute, and the sum
// is bit-identical in the four lanes of a row.
// (The max as compare and select: fmaxf cannot tell that the swapped bits are
// canonical and quiets both operands first, three instructions instead of two.
// Scores are never NaN here: masked keys carry -1e30.)
__device__ __forceinline__ float max_pair(float a, float b) { return a > b ? a : b; }
__device__ __forceinline__ float lane_groups_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = max_pair(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_pair(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float lane_groups_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 2^x with the hardware exponential alone (v_exp_f32).  exp2f adds a range
// reduction that keeps results below 2^-126 as denormals (six instructions
// instead of one); a softmax never needs them: every probability is
// 2^(score - m) with the row's running max m at most 2^8 below its largest
// score, so a term under 2^-126 is below 2^-134 of the row's sum and its
// flush to zero changes nothing, and masked scores (-1e30) give exactly 0.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Called by the whole wave when some lane holds a score above its row's
// threshold: each row takes its max over its four lane groups and raises m to
// it if that exceeds m by more than kLazyMax, rescaling its output and sum.
// The first step of every row comes here (thr starts at kNegBig and every row
// has a key in its first step).
template <int NO>
__device__ __forceinline__ void raise_max(RowState& r, float mx, float scale_log2, float inv_scale,
                                          f32x4 (&o)[NO]) {
  const float rmx = lane_groups_max(mx) * scale_log2;  // scale > 0: the max of the scaled scores
  const bool raise = rmx > r.m + kLazyMax;
  const float m_new = raise ? rmx : r.m;
  const float alpha = raise ? fast_exp2(r.m - m_new) : 1.f;
#pragma unroll
  for (int e = 0; e < NO; e++) o[e] = o[e] * alpha;
  r.l *= alpha;
  r.m = m_new;
  r.thr = (m_new + kLazyMax) * inv_scale;
}

// v[e] = the 16 bytes at LDS address addr + OFF0 + e * STEP, e = E .. N - 1.
template <int E, int N, int OFF0, int STEP>
__device__ __forceinline__ void lds_read_run(unsigned addr, u32x4 (&v)[N]) {
  if constexpr (E < N) {
    v[E] = lds_read16_at<OFF0 + E * STEP>(addr);
    lds_read_run<E + 1, N, OFF0, STEP>(addr, v);
  }
}

// Deterministic merge of the key splits of one (decode request, q head), a
// workgroup each: HD / 4 threads hold a split's row, so 8 (HD = 128) or 16 splits
// are read side by side, every load independent of the others (running maximum
// per thread, the groups' states combined through LDS in group order).  Bound by
// latency: 4.5 us for 33 splits (70B heads, four requests), where one thread per
// dim that walked the splits twice in turn took 13.3 us.
constexpr int kMergeThreads = 256;
template <int HD>
constexpr int merge_floats() {
  return kMergeThreads / (HD / 4) * (HD + 2);
}
template <int HD>
__device__ __forceinline__ void merge_splits(const AttnParams& p, const MergeItem& mi, int h,
                                             float* smem) {
  constexpr int TPR = HD / 4, G = kMergeThreads / TPR;
  float(*s_acc)[HD] = reinterpret_cast<float(*)[HD]>(smem);
  float *s_m = smem + G * HD, *s_l = s_m + G;
  const ReqDev rq = p.reqs[mi.req];
  const int g = threadIdx.x / TPR, d = 4 * (threadIdx.x % TPR);
  const int ns = rq.n_split;
  const int64_t base = (int64_t)mi.part_base + (int64_t)h * ns;
  float m = kNegBig, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = g; s < ns; s += G) {
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (base + s) * 2);
    const f32x4 o = *reinterpret_cast<const f32x4*>(p.part_o + (base + s) * HD + d);
    const float mn = fmaxf(m, ml.x);
    const float a = exp2f(m - mn), w = exp2f(ml.x - mn);
    acc = acc * a + o * w;
    l = l * a + ml.y * w;
    m = mn;
  }
  *reinterpret_cast<f32x4*>(&s_acc[g][d]) = acc;
  if (d == 0) {
    s_m[g] = m;
    s_l[g] = l;
  }
  __syncthreads();
  if (threadIdx.x >= HD / 2) return;
  float M = kNegBig;
#pragma unroll
  for (int k = 0; k < G; k++) M = fmaxf(M, s_m[k]);
  float L = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
  for (int k = 0; k < G; k++) {
    const float w = exp2f(s_m[k] - M);  // a group without a split: 0 (some split has a key)
    L += s_l[k] * w;
    a0 += s_acc[k][2 * threadIdx.x] * w;
    a1 += s_acc[k][2 * threadIdx.x + 1] * w;
  }
  *reinterpret_cast<uint32_t*>(out_ptr(p, rq.tok_start, h * HD + 2 * threadIdx.x)) =
      pack_bf16x2(a0 / L, a1 / L);
}

}  // namespace

}  // namespace mx
