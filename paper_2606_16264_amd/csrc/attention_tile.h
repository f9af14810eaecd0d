// attention_tile.h -- what the attention kernels share: the output's address, the
// online softmax of a query row held by four lanes, runs of LDS fragment reads.
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

}  // namespace

}  // namespace mx
