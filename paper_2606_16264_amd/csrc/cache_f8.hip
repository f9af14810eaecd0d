// cache_f8.hip -- the 8-bit key/value cache's append and its eviction by accumulated
// attention weight on gfx950.
//
// A page holds 16 tokens of every KV head as e4m3 codes, with one power-of-two scale
// for its keys and one for its values per head: the code of x is x / scale rounded
// to nearest even.  Powers of two make x / scale exact, so a code is one rounding away
// from its value, and a page's codes move to a larger scale by a shift of their
// exponents (exact unless they end below the smallest normal code).
#include "mx_device.h"
#include "mx_kernels.h"

namespace mx {

namespace {

// The least power of two 2^e with amax <= 448 2^e (448: the largest code), e clamped
// to [-100, 119]: below, everything to 2^-109 still has a code; above, the largest
// code stands for 1.75 * 2^127, which fp32 and bf16 hold.
__device__ __forceinline__ float fit_scale(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000);
  return __uint_as_float((uint32_t)(min(max(e, -100), 119) + 127) << 23);
}
// 1 / scale of a power of two: the exponent negated.
__device__ __forceinline__ float inverse(float scale) {
  return __uint_as_float((254u << 23) - __float_as_uint(scale));
}
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < __builtin_inff(); }
__device__ __forceinline__ float max_finite(float m, float x) {
  return finite(x) ? fmaxf(m, __builtin_fabsf(x)) : m;
}

// Two values over the scale as codes in the low half; what is not finite becomes NaN
// (0x7F), what a clamped scale leaves beyond the largest code becomes that.
__device__ __forceinline__ uint32_t encode2(float a, float b, float inv) {
  const float x = __builtin_amdgcn_fmed3f(a * inv, -448.f, 448.f);
  const float y = __builtin_amdgcn_fmed3f(b * inv, -448.f, 448.f);
  const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xFFFFu;
  return (finite(a) ? c & 0xFFu : 0x7Fu) | (finite(b) ? c & 0xFF00u : 0x7F00u);
}
// Four codes times a power of two at most 1, as codes; NaN codes stay as they are (the
// conversions would change their bits).
__device__ __forceinline__ uint32_t shift_codes(uint32_t c, float ratio) {
  const mx_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false);
  const mx_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio, lo[1] * ratio, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio, hi[1] * ratio, r, true);
  // (a byte's low seven bits plus one reach its top bit for NaN alone)
  const uint32_t nan = ((((c & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u) * 0xFFu;
  return ((uint32_t)r & ~nan) | (c & nan);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The page's scale with the new tokens in it: never below that of the older tokens
// that stay, which move to the new one (ratio = old / new, 1 where it did not change).
struct PageScale {
  float now, ratio;
};
__device__ __forceinline__ PageScale page_scale(float amax, const float* scale, int s0) {
  const float need = fit_scale(amax);
  const float old = s0 > 0 ? *scale : 0.f;
  return old >= need ? PageScale{old, 1.f} : PageScale{need, old * inverse(need)};
}

// ---------------------------------------------------------------- append
// One wave per (run, KV head, keys or values): the up to 16 new tokens of one page.
// Keys: 16 lanes (HD = 128) or 8 hold a token, 8 dims each, and write the 8 codes to
// the page's 64-dim block.  Values: a lane holds HD / 64 dims of every token and
// writes whole 16-byte rows of the transposed page, in which the bytes of other
// tokens are put back as they were.
template <int HD>
__device__ __forceinline__ void append_keys(const uint16_t* __restrict__ src, int64_t row,
                                            uint8_t* __restrict__ dst, float* __restrict__ scale,
                                            float* __restrict__ weight, int s0, int n, int lane) {
  constexpr int TPR = HD / 8, RPI = 64 / TPR, NI = 16 / RPI;  // lanes per token, tokens per load
  const int c = lane % TPR;
  u32x4 x[NI];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < NI; i++) {
    const int t = i * RPI + lane / TPR;
    x[i] = t < n ? *reinterpret_cast<const u32x4*>(src + t * row + 8 * c) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; e++) amax = max_finite(max_finite(amax, lo_f32(x[i][e])), hi_f32(x[i][e]));
  }
  const PageScale ps = page_scale(wave_max(amax), scale, s0);
  const float inv = inverse(ps.now);
  uint8_t* d = dst + (c >> 3) * 1024 + (c & 7) * 8;
#pragma unroll
  for (int i = 0; i < NI; i++) {
    const int t = i * RPI + lane / TPR;
    if (t < n) {
      u32x2 w;
      w[0] = encode2(lo_f32(x[i][0]), hi_f32(x[i][0]), inv) |
             encode2(lo_f32(x[i][1]), hi_f32(x[i][1]), inv) << 16;
      w[1] = encode2(lo_f32(x[i][2]), hi_f32(x[i][2]), inv) |
             encode2(lo_f32(x[i][3]), hi_f32(x[i][3]), inv) << 16;
      *reinterpret_cast<u32x2*>(d + (s0 + t) * 64) = w;
    }
    if (ps.ratio != 1.f && t < s0) {
      u32x2 w = *reinterpret_cast<u32x2*>(d + t * 64);
      w[0] = shift_codes(w[0], ps.ratio);
      w[1] = shift_codes(w[1], ps.ratio);
      *reinterpret_cast<u32x2*>(d + t * 64) = w;
    }
  }
  if (lane == 0) *scale = ps.now;
  if (weight && lane < n) weight[s0 + lane] = 0.f;
}

template <int HD>
__device__ __forceinline__ void append_values(const uint16_t* __restrict__ src, int64_t row,
                                              uint8_t* __restrict__ dst, float* __restrict__ scale,
                                              int s0, int n, int lane) {
  constexpr int ND = HD / 64;  // dims per lane: ND lane .. + ND - 1
  float x[16][ND];
  float amax = 0.f;
#pragma unroll
  for (int t = 0; t < 16; t++) {
    uint32_t w = 0;
    if (t < n) {
      if constexpr (ND == 2) w = *reinterpret_cast<const uint32_t*>(src + t * row + 2 * lane);
      else w = src[t * row + lane];
    }
    x[t][0] = lo_f32(w);
    if constexpr (ND == 2) x[t][1] = hi_f32(w);
#pragma unroll
    for (int e = 0; e < ND; e++) amax = max_finite(amax, x[t][e]);
  }
  const PageScale ps = page_scale(wave_max(amax), scale, s0);
  const float inv = inverse(ps.now);
#pragma unroll
  for (int e = 0; e < ND; e++) {
    u32x4* d = reinterpret_cast<u32x4*>(dst + (ND * lane + e) * 16);
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; q++)
      w[q] = encode2(x[4 * q][e], x[4 * q + 1][e], inv) |
             encode2(x[4 * q + 2][e], x[4 * q + 3][e], inv) << 16;
    if (n < 16) {
      // token t's code goes to byte s0 + t; the bytes before it are older tokens'
      u32x4 old = *d;
      const unsigned __int128 all = (unsigned __int128)-1;
      unsigned __int128 nw = __builtin_bit_cast(unsigned __int128, w) << (8 * s0);
      const unsigned __int128 mask = (all >> (8 * (16 - n))) << (8 * s0);
      if (ps.ratio != 1.f) {
        const unsigned __int128 before = s0 > 0 ? all >> (8 * (16 - s0)) : 0;
        u32x4 sh;
#pragma unroll
        for (int q = 0; q < 4; q++) sh[q] = shift_codes(old[q], ps.ratio);
        old = __builtin_bit_cast(u32x4, (__builtin_bit_cast(unsigned __int128, sh) & before) |
                                            (__builtin_bit_cast(unsigned __int128, old) & ~before));
      }
      w = __builtin_bit_cast(u32x4, (nw & mask) | (__builtin_bit_cast(unsigned __int128, old) & ~mask));
    }
    *d = w;
  }
  if (lane == 0) *scale = ps.now;
}

template <int HD>
__global__ __launch_bounds__(256) void kv_append_f8_kernel(const uint16_t* __restrict__ k_new,
                                                           const uint16_t* __restrict__ v_new,
                                                           CacheF8 c, const AppendRun* runs,
                                                           int nkv) {
  const u32x4 rw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(runs + blockIdx.x));
  const AppendRun run = __builtin_bit_cast(AppendRun, rw);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.y * 4 + wave;  // 2 g: keys of head g, 2 g + 1: its values
  if (unit >= 2 * nkv) return;
  const int g = unit >> 1, s0 = (int)(run.slot & 15);
  const int64_t at = (run.slot >> 4) * nkv + g, row = (int64_t)nkv * HD;
  const int64_t src = run.tok * row + (int64_t)g * HD;
  if ((unit & 1) == 0)
    append_keys<HD>(k_new + src, row, c.k + at * (16 * HD), c.k_scale + at,
                    c.weight ? c.weight + at * 16 : nullptr, s0, run.n, lane);
  else
    append_values<HD>(v_new + src, row, c.v + at * (16 * HD), c.v_scale + at, s0, run.n, lane);
}

// ---------------------------------------------------------------- eviction
// An order-preserving map of fp32 weights to unsigned integers (-0 as 0).
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
  return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

constexpr int kSelectThreads = 1024;

// One workgroup per (request, KV head): the threshold of the (keep - recent) largest
// weights among the first len - recent tokens by radix selection, 8 bits a pass from
// the top, then the kept tokens' indices in order.  Of the tokens at the threshold
// the first ones are kept.
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(
    const EvictReq* reqs, const int32_t* pages, const float* __restrict__ weight, int nkv,
    int32_t* __restrict__ kept) {
  __shared__ uint32_t s_hist[256];
  __shared__ uint32_t s_pick[2];  // digit, rank left within it
  __shared__ uint32_t s_cnt[2][kSelectThreads / 64];
  const EvictReq rq = reqs[blockIdx.x];
  const int g = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int32_t* ptab = pages + rq.src;
  auto key = [&](int j) {
    return weight_key(weight[((int64_t)ptab[j >> 4] * nkv + g) * 16 + (j & 15)]);
  };
  const int n = rq.len - rq.recent;
  const uint32_t want = rq.keep - rq.recent;
  uint32_t thr = 0, left = want;  // left: how many of the tokens at the threshold stay
  if (want > 0 && want < (uint32_t)n) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = t; i < 256; i += kSelectThreads) s_hist[i] = 0;
      __syncthreads();
      for (int j = t; j < n; j += kSelectThreads) {
        const uint32_t k = key(j);
        if (shift == 24 || (k >> (shift + 8)) == (thr >> (shift + 8)))
          atomicAdd(&s_hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (t == 0) {
        uint32_t above = 0;
        int dig = 255;
        while (above + s_hist[dig] < left) above += s_hist[dig--];
        s_pick[0] = dig;
        s_pick[1] = left - above;
      }
      __syncthreads();
      thr |= s_pick[0] << shift;
      left = s_pick[1];
    }
  }
  int32_t* out = kept + rq.kept + (int64_t)g * rq.keep;
  uint32_t done = 0, ties = 0;
  const uint64_t below = (1ull << lane) - 1;
  if (want > 0) {
    for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
      const int j = j0 + t;
      const uint32_t k = j < n ? key(j) : 0u;
      // (want == n: thr is 0 and left is n, so that every token stays)
      const bool gt = j < n && want < (uint32_t)n && k > thr;
      const bool eq = j < n && (want == (uint32_t)n || k == thr);
      const uint64_t bg = __ballot(gt), be = __ballot(eq);
      if (lane == 0) {
        s_cnt[0][wave] = __popcll(bg);
        s_cnt[1][wave] = __popcll(be);
      }
      __syncthreads();
      uint32_t g0 = 0, e0 = 0, gall = 0, eall = 0;
      for (int w = 0; w < kSelectThreads / 64; w++) {
        if (w < wave) g0 += s_cnt[0][w], e0 += s_cnt[1][w];
        gall += s_cnt[0][w];
        eall += s_cnt[1][w];
      }
      g0 += __popcll(bg & below);
      e0 += ties + __popcll(be & below);
      // kept ties ahead of this token: those of the first `left` ties with a lower index
      const uint32_t at = done + g0 + (min(e0, left) - min(ties, left));
      if (gt || (eq && e0 < left)) out[at] = j;
      done += gall + (min(ties + eall, left) - min(ties, left));
      ties += eall;
      __syncthreads();
    }
  }
  for (int i = t; i < rq.recent; i += kSelectThreads) out[want + i] = n + i;
}

// Copies the kept tokens of one destination page and KV head, a wave each.  The page's
// scale is the largest of those its tokens come from.
template <int HD>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictReq* reqs,
                                                         const int32_t* pages,
                                                         const EvictPage* items, CacheF8 c, int nkv,
                                                         const int32_t* __restrict__ kept) {
  const EvictPage it = items[blockIdx.x];
  const EvictReq rq = reqs[it.req];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int g = blockIdx.y * 4 + wave;
  if (g >= nkv) return;
  const int n = min(16, rq.keep - it.start);  // tokens of this page
  const int64_t dst = (int64_t)pages[rq.dst + (it.start >> 4)] * nkv + g;
  // token i of the page lives at lanes i, i + 16 ..: its source page and slot, and scales
  const int ti = min(lane & 15, n - 1);
  const int j = kept[rq.kept + (int64_t)g * rq.keep + it.start + ti];
  const int64_t src = (int64_t)pages[rq.src + (j >> 4)] * nkv + g;
  const int slot = j & 15;
  float ks = c.k_scale[src], vs = c.v_scale[src];
  float kn = ks, vn = vs;
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) {
    kn = fmaxf(kn, __shfl_xor(kn, m));
    vn = fmaxf(vn, __shfl_xor(vn, m));
  }
  const float kr = ks * inverse(kn), vr = vs * inverse(vn);
  if (lane == 0) {
    c.k_scale[dst] = kn;
    c.v_scale[dst] = vn;
  }
  if (lane < n) c.weight[dst * 16 + lane] = c.weight[src * 16 + slot];
  // keys: 16 bytes per lane in the destination's order
#pragma unroll
  for (int q = 0; q < HD / 64; q++) {
    const int i = lane >> 2, from = min(i, n - 1);
    const int64_t sp = __shfl(src, from);
    const int ss = __shfl(slot, from);
    const float ratio = __shfl(kr, from);
    if (i < n) {
      u32x4 w = *reinterpret_cast<const u32x4*>(c.k + sp * (16 * HD) + q * 1024 + ss * 64 + (lane & 3) * 16);
      if (ratio != 1.f)
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = shift_codes(w[e], ratio);
      *reinterpret_cast<u32x4*>(c.k + dst * (16 * HD) + q * 1024 + i * 64 + (lane & 3) * 16) = w;
    }
  }
  // values: a lane's rows of the transposed page, gathered byte by byte
#pragma unroll
  for (int q = 0; q < HD / 64; q++) {
    const int e = q * 64 + lane;
    u32x4* d = reinterpret_cast<u32x4*>(c.v + dst * (16 * HD) + e * 16);
    u32x4 w = n < 16 ? *d : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const int64_t sp = __shfl(src, i);
      const int ss = __shfl(slot, i);
      const float ratio = __shfl(vr, i);
      if (i < n) {
        uint32_t b = c.v[sp * (16 * HD) + e * 16 + ss];
        if (ratio != 1.f) b = shift_codes(b, ratio) & 0xFFu;
        w[i >> 2] = (w[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | b << (8 * (i & 3));
      }
    }
    *d = w;
  }
}

}  // namespace

hipError_t launch_kv_append_f8(const uint16_t* k_new, const uint16_t* v_new, const CacheF8& cache,
                               const AppendRun* runs, int64_t n_runs, int nkv, int d,
                               hipStream_t stream) {
  if (n_runs == 0) return hipSuccess;
  const dim3 grid((unsigned)n_runs, (2 * nkv + 3) / 4);
  if (d == 128)
    kv_append_f8_kernel<128><<<grid, 256, 0, stream>>>(k_new, v_new, cache, runs, nkv);
  else
    kv_append_f8_kernel<64><<<grid, 256, 0, stream>>>(k_new, v_new, cache, runs, nkv);
  return hipGetLastError();
}

hipError_t launch_kv_evict_f8(const EvictReq* reqs, int n_reqs, const int32_t* pages,
                              const EvictPage* items, int64_t n_items, const CacheF8& cache,
                              int32_t* kept, int nkv, int d, hipStream_t stream) {
  if (n_items == 0) return hipSuccess;
  evict_select_kernel<<<dim3(n_reqs, nkv), kSelectThreads, 0, stream>>>(reqs, pages, cache.weight,
                                                                       nkv, kept);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)n_items, (nkv + 3) / 4);
  if (d == 128)
    evict_move_kernel<128><<<grid, 256, 0, stream>>>(reqs, pages, items, cache, nkv, kept);
  else
    evict_move_kernel<64><<<grid, 256, 0, stream>>>(reqs, pages, items, cache, nkv, kept);
  return hipGetLastError();
}

}  // namespace mx
