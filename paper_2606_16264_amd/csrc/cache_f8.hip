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
// Four codes times powers of two at most 1, as codes; NaN codes stay as they are (the
// conversions would change their bits).  down: eight times the exponents' decrease, a
// byte per code (at most 120 each, which any larger one is given as).  Where every code
// stays normal its exponent field is lowered in place; else the codes go through fp32,
// times ratio[i] = 2^-decrease, and round to nearest even.
__device__ __forceinline__ uint32_t shift_codes(uint32_t c, uint32_t down, const float (&ratio)[4]) {
  const uint32_t mag = c & 0x7F7F7F7Fu;
  // a byte's top bit: magnitude at least 8 * (decrease + 1); NaN, 0x7F plus one
  const uint32_t normal = (mag + (0x80808080u - 0x08080808u - down)) & 0x80808080u;
  const uint32_t nan = (mag + 0x01010101u) & 0x80808080u;
  if (normal == 0x80808080u && nan == 0) return c - down;
  const mx_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false);
  const mx_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio[0], lo[1] * ratio[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio[2], hi[1] * ratio[3], r, true);
  const uint32_t keep = (nan >> 7) * 0xFFu;
  return ((uint32_t)r & ~keep) | (c & keep);
}
// How far the exponent of a power of two lies below another's, capped as shift_codes
// takes it.
__device__ __forceinline__ int exponent_drop(float from, float to) {
  return min(max((int)(__float_as_uint(to) >> 23) - (int)(__float_as_uint(from) >> 23), 0), 15);
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
  uint32_t down;  // ratio as shift_codes takes it, all four bytes alike

  __device__ __forceinline__ uint32_t shift(uint32_t c) const {
    const float r[4] = {ratio, ratio, ratio, ratio};
    return shift_codes(c, down, r);
  }
};
__device__ __forceinline__ PageScale page_scale(float amax, const float* scale, int s0) {
  const float need = fit_scale(amax);
  const float old = s0 > 0 ? *scale : 0.f;
  if (old >= need) return PageScale{old, 1.f, 0};
  return PageScale{need, old * inverse(need), exponent_drop(old, need) * 0x08080808u};
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
      w[0] = ps.shift(w[0]);
      w[1] = ps.shift(w[1]);
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
        for (int q = 0; q < 4; q++) sh[q] = ps.shift(old[q]);
        old = __builtin_bit_cast(u32x4, (__builtin_bit_cast(unsigned __int128, sh) & before) |
                                            (__builtin_bit_cast(unsigned __int128, old) & ~before));
      }
      w = __builtin_bit_cast(u32x4, (nw & mask) | (__builtin_bit_cast(unsigned __int128, old) & ~mask));
    }
    *d = w;
  }
  if (lane == 0) *scale = ps.now;
}

// This wave's unit of a run: 2 g is the keys of head g, 2 g + 1 its values.
template <int HD>
__device__ __forceinline__ void append_unit(const uint16_t* k_new, const uint16_t* v_new,
                                            const CacheF8& c, const AppendRun& run, int nkv) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.y * 4 + wave;
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

template <int HD>
__global__ __launch_bounds__(256) void kv_append_f8_kernel(const uint16_t* k_new,
                                                           const uint16_t* v_new, CacheF8 c,
                                                           const AppendRun* runs, int nkv) {
  const u32x4 rw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(runs + blockIdx.x));
  append_unit<HD>(k_new, v_new, c, __builtin_bit_cast(AppendRun, rw), nkv);
}

struct SmallAppend {
  const uint16_t *k_new, *v_new;
  CacheF8 c;
  int64_t nkv;
  InlineMeta runs;
};
template <int HD>
__global__ __launch_bounds__(256) void small_append_f8_kernel(SmallAppend a) {
  const AppendRun* runs = inline_meta<AppendRun>(offsetof(SmallAppend, runs), nullptr);
  append_unit<HD>(a.k_new, a.v_new, a.c, runs[blockIdx.x], (int)a.nkv);
}

// ---------------------------------------------------------------- eviction
// An order-preserving map of fp32 weights to unsigned integers: -0 as 0, every NaN, of
// either sign, as the largest.  (Selects on integers: float comparisons became branches,
// between which a thread's loads went one by one, 28 us for evict_select's 16.)
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w), mag = b & 0x7FFFFFFFu;
  const uint32_t key = b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
  return mag > 0x7F800000u ? ~0u : mag == 0 ? 0x80000000u : key;
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// Sum of x over this lane and the ones above it in the wave.
__device__ __forceinline__ uint32_t suffix_sum(uint32_t x, int lane) {
  // within rows of 16 lanes: lane i adds lane i + 1, + 2, + 4, + 8 (0 past the row)
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x101, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x102, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x104, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x108, 0xF, 0xF, true);
  const uint32_t r1 = __builtin_amdgcn_readlane(x, 16), r2 = __builtin_amdgcn_readlane(x, 32),
                 r3 = __builtin_amdgcn_readlane(x, 48);
  const int row = lane >> 4;
  return x + (row == 0 ? r1 + r2 + r3 : row == 1 ? r2 + r3 : row == 2 ? r3 : 0u);
}

// One workgroup per (request, KV head).  Among the first n = len - recent tokens the
// want = keep - recent with the largest keys stay, of equal ones the first.
//
// The want-th largest key is found eight bits at a time from the top, by a histogram in
// LDS of the keys that agree with it so far.  Most weights share their exponent and many
// are zero, and adds of one wave to one counter go in turn, so a digit has four counters,
// of which a lane takes the one of its own index (16 requests of up to 16384 tokens, 8
// heads: 16 us; counting up to 16 times the keys at or above three candidates by
// ballots, 38).  The search ends early when a digit's keys are just what is missing.
// Each wave holds 64 K consecutive tokens, K a lane in registers (K = 0: any number,
// read again in every pass), so the kept indices need one scan over the waves.  Bound
// by latency: loads, then up to four times adds, a barrier, the scan of the counters by
// one wave, a barrier.
template <int K>
__device__ __forceinline__ void evict_select(const EvictReq* reqs, const int32_t* pages,
                                             const float* __restrict__ weight, int nkv,
                                             int32_t* __restrict__ kept) {
  __shared__ __attribute__((aligned(16))) uint32_t s_hist[4][256][4];
  __shared__ uint32_t s_pick[4][3];  // digit, keys missing within it, keys of it
  __shared__ __attribute__((aligned(16))) uint32_t s_total[kSelectWaves][2];
  const EvictReq rq = reqs[blockIdx.x];
  const int g = blockIdx.y, t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int32_t* ptab = pages + rq.src;
  const int n = rq.len - rq.recent;
  const uint32_t want = rq.keep - rq.recent;
  const int per = K > 0 ? K : (n + kSelectThreads - 1) / kSelectThreads;  // 64-token groups per wave
  const int first = wave * per * 64 + lane;
  auto load = [&](int i) -> uint32_t {
    // (past the end: 0, below every candidate; the load itself is unconditional, so that
    // a thread's loads are in flight together)
    const int j = first + 64 * i, jc = min(j, n - 1);
    const uint32_t k = weight_key(weight[((int64_t)ptab[jc >> 4] * nkv + g) * 16 + (jc & 15)]);
    return j < n ? k : 0u;
  };
  int32_t* out = kept + rq.kept + (int64_t)g * rq.keep;
  for (int i = t; i < rq.recent; i += kSelectThreads) out[want + i] = n + i;
  if (want == 0) return;
  uint32_t held[K > 0 ? K : 1];
  if constexpr (K > 0) {
#pragma unroll
    for (int i = 0; i < K; i++) held[i] = load(i);
  }
  auto each = [&](auto f) {  // f(64-token group, its keys)
    if constexpr (K > 0) {
#pragma unroll
      for (int i = 0; i < K; i++) f(i, held[i]);
    } else {
      for (int i = 0; i < per; i++) f(i, load(i));
    }
  };

  // keys above thr stay, and the first `left` of those equal to it
  uint32_t thr = 0;
  const bool all = want >= (uint32_t)n;
  if (!all) {
    reinterpret_cast<u32x4*>(s_hist)[t] = u32x4{0, 0, 0, 0};
    __syncthreads();
    uint32_t missing = want;  // keys to take among those that agree with thr so far
#pragma unroll 1
    for (int pass = 0; pass < 4; pass++) {
      const int shift = 24 - 8 * pass;
      // (pass 0: every key agrees with none of its bits)
      const uint32_t fixed = pass == 0 ? 0u : ~0u << (shift + 8);
      each([&](int i, uint32_t k) {
        if (first + 64 * i < n && ((k ^ thr) & fixed) == 0)
          atomicAdd(&s_hist[pass][k >> shift & 255][lane & 3], 1u);
      });
      __syncthreads();
      if (wave == 0) {
        uint32_t h[4], mine = 0;  // digits 4 lane .. 4 lane + 3
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const u32x4 c = *reinterpret_cast<const u32x4*>(s_hist[pass][4 * lane + e]);
          h[e] = (c[0] + c[1]) + (c[2] + c[3]);
          mine += h[e];
        }
        uint32_t above = suffix_sum(mine, lane) - mine;  // keys of larger digits
#pragma unroll
        for (int e = 3; e >= 0; e--) {
          if (above < missing && missing <= above + h[e]) {  // one digit of one lane
            s_pick[pass][0] = 4 * lane + e;
            s_pick[pass][1] = missing - above;
            s_pick[pass][2] = h[e];
          }
          above += h[e];
        }
      }
      __syncthreads();
      thr |= (uint32_t)__builtin_amdgcn_readfirstlane(s_pick[pass][0]) << shift;
      missing = __builtin_amdgcn_readfirstlane(s_pick[pass][1]);
      if (missing == (uint32_t)__builtin_amdgcn_readfirstlane(s_pick[pass][2])) {
        thr--;  // every key from here on stays; want < n, so some key is below thr, which is not 0
        break;
      }
    }
  }
  uint32_t above = 0, equal = 0;
  each([&](int i, uint32_t k) {  // per lane; a ballot each took four times as long
    const bool in = first + 64 * i < n;
    above += in && (all || k > thr);
    equal += in && !all && k == thr;
  });
  above = suffix_sum(above, lane);
  equal = suffix_sum(equal, lane);
  if (lane == 0) {
    s_total[wave][0] = above;
    s_total[wave][1] = equal;
  }
  __syncthreads();
  uint32_t done = 0, ties = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; w++) {
    const uint32_t a = __builtin_amdgcn_readfirstlane(s_total[w][0]);
    const uint32_t e = __builtin_amdgcn_readfirstlane(s_total[w][1]);
    total += a;
    done += w < wave ? a : 0;
    ties += w < wave ? e : 0;
  }
  const uint32_t left = want - total;
  done += min(ties, left);
  const uint64_t below = (1ull << lane) - 1;
  each([&](int i, uint32_t k) {
    const int j = first + 64 * i;
    const bool gt = j < n && (all || k > thr), eq = j < n && !all && k == thr;
    const uint64_t bg = __ballot(gt), be = left ? __ballot(eq) : 0;
    const uint32_t tie = ties + __popcll(be & below);
    if (gt || (eq && tie < left))
      out[done + __popcll(bg & below) + min(tie, left) - min(ties, left)] = j;
    const uint32_t next = ties + __popcll(be);
    done += __popcll(bg) + min(next, left) - min(ties, left);
    ties = next;
  });
}

template <int K>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictReq* reqs,
                                                                      const int32_t* pages,
                                                                      const float* weight, int nkv,
                                                                      int32_t* kept) {
  evict_select<K>(reqs, pages, weight, nkv, kept);
}

// Copies the kept tokens of one destination page and KV head, a wave each.  The page's
// scale is the largest of those its tokens come from.  Bound by memory: 108 us for up to
// 8192 tokens each of 16 requests, 8 heads, 623 MB (190 written; keys are 64-byte runs,
// and of a value page that holds one kept token all lines are read, since a token's
// values lie 16 bytes apart).  Values: the tokens of a destination page come from source
// pages in ascending order; of each such page a lane reads its rows as 16-byte words
// and takes the bytes it needs with byte permutes whose selectors are the same in all
// lanes (as loads of single bytes: 177 us).
template <int HD>
__device__ __forceinline__ void evict_move(const EvictReq* reqs, const int32_t* pages,
                                           const EvictPage* items, const CacheF8& c, int nkv,
                                           const int32_t* __restrict__ kept) {
  constexpr int NR = HD / 64;  // value rows per lane: lane, lane + 64
  const EvictPage it = items[blockIdx.x];
  const EvictReq rq = reqs[it.req];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = blockIdx.y * 4 + wave;
  if (g >= nkv) return;
  const int n = min(16, rq.keep - it.start);  // tokens of this page
  const int64_t dst = (int64_t)pages[rq.dst + (it.start >> 4)] * nkv + g;
  // token i of the page lives at lanes i, i + 16 ..: its source page and slot, and scales
  const int ti = min(lane & 15, n - 1);
  const int j = kept[rq.kept + (int64_t)g * rq.keep + it.start + ti];
  const int page = pages[rq.src + (j >> 4)], slot = j & 15;
  const int64_t src = (int64_t)page * nkv + g;
  const float ks = c.k_scale[src], vs = c.v_scale[src];
  float kn = ks, vn = vs;
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) {
    kn = fmaxf(kn, __shfl_xor(kn, m));
    vn = fmaxf(vn, __shfl_xor(vn, m));
  }
  if (lane == 0) {
    c.k_scale[dst] = kn;
    c.v_scale[dst] = vn;
  }
  if (lane < n) c.weight[dst * 16 + lane] = c.weight[src * 16 + slot];

  // the first source page's values, on their way while the keys are copied
  const int before = __shfl_up(page, 1);
  uint32_t starts = (uint32_t)__ballot(lane < n && (lane == 0 || page != before));
  auto rows = [&](int i, u32x4 (&r)[NR]) {  // value rows of token i's page
    const int64_t at = (int64_t)__builtin_amdgcn_readlane(page, i) * nkv + g;
#pragma unroll
    for (int q = 0; q < NR; q++)
      r[q] = *reinterpret_cast<const u32x4*>(c.v + at * (16 * HD) + q * 1024 + lane * 16);
  };
  u32x4 r[NR], next[NR];
  rows(0, r);

  // keys: 16 bytes per lane in the destination's order, token lane / 4
  {
    const int i = min(lane >> 2, n - 1);
    const int64_t sp = (int64_t)__shfl(page, i) * nkv + g;
    const int ss = __shfl(slot, i);
    const float from = __shfl(ks, i), ratio = from * inverse(kn);
    const uint32_t down = exponent_drop(from, kn) * 0x08080808u;
    const float all[4] = {ratio, ratio, ratio, ratio};
    const uint8_t* s = c.k + sp * (16 * HD) + ss * 64 + (lane & 3) * 16;
    uint8_t* d = c.k + dst * (16 * HD) + lane * 16;
    u32x4 w[NR];
#pragma unroll
    for (int q = 0; q < NR; q++) w[q] = *reinterpret_cast<const u32x4*>(s + q * 1024);
    if (down) {
#pragma unroll
      for (int q = 0; q < NR; q++)
#pragma unroll
        for (int e = 0; e < 4; e++) w[q][e] = shift_codes(w[q][e], down, all);
    }
    if ((lane >> 2) < n) {
#pragma unroll
      for (int q = 0; q < NR; q++) *reinterpret_cast<u32x4*>(d + q * 1024) = w[q];
    }
  }

  // values: the words of the destination rows, bytes of one source page at a time
  u32x4 w[NR];
#pragma unroll
  for (int q = 0; q < NR; q++) w[q] = u32x4{0, 0, 0, 0};
  auto quad = [&](uint32_t byte) {  // lanes 4 q .. 4 q + 3's bytes as one word
    uint32_t x = byte << (8 * (lane & 3));
    x |= __builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
    x |= __builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true);   // lanes 2 3 0 1
    return x;
  };
  while (starts) {
    const int i0 = __builtin_ctz(starts);
    starts &= starts - 1;
    const int i1 = starts ? __builtin_ctz(starts) : n;
    if (starts) rows(i1, next);
    // selector 12 is a zero byte
    const bool mine = lane >= i0 && lane < i1;
    const uint32_t lo = quad(mine && slot < 8 ? slot : 12), hi = quad(mine && slot >= 8 ? slot - 8 : 12);
#pragma unroll
    for (int d = 0; d < 4; d++) {
      const uint32_t sl = __builtin_amdgcn_readlane(lo, 4 * d), sh = __builtin_amdgcn_readlane(hi, 4 * d);
#pragma unroll
      for (int q = 0; q < NR; q++)
        w[q][d] |= __builtin_amdgcn_perm(r[q][1], r[q][0], sl) | __builtin_amdgcn_perm(r[q][3], r[q][2], sh);
    }
#pragma unroll
    for (int q = 0; q < NR; q++) r[q] = next[q];
  }
  const float ratio = vs * inverse(vn);
  const int drop = 8 * exponent_drop(vs, vn);
  if (__any(drop)) {
    const uint32_t down = quad(drop);
#pragma unroll
    for (int d = 0; d < 4; d++) {
      const uint32_t dd = __builtin_amdgcn_readlane(down, 4 * d);
      float by[4];
#pragma unroll
      for (int e = 0; e < 4; e++)
        by[e] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ratio), 4 * d + e));
      if (dd)
#pragma unroll
        for (int q = 0; q < NR; q++) w[q][d] = shift_codes(w[q][d], dd, by);
    }
  }
#pragma unroll
  for (int q = 0; q < NR; q++) {
    u32x4* d = reinterpret_cast<u32x4*>(c.v + dst * (16 * HD) + q * 1024 + lane * 16);
    if (n < 16) {  // the bytes behind the page's tokens stay
      const u32x4 old = *d;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int b = min(max(n - 4 * e, 0), 4);
        const uint32_t mask = b == 4 ? ~0u : (1u << (8 * b)) - 1;
        w[q][e] = (w[q][e] & mask) | (old[e] & ~mask);
      }
    }
    *d = w[q];
  }
}

template <int HD>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictReq* reqs,
                                                         const int32_t* pages,
                                                         const EvictPage* items, CacheF8 c, int nkv,
                                                         const int32_t* kept) {
  evict_move<HD>(reqs, pages, items, c, nkv, kept);
}

struct SmallEvict {
  const EvictReq* reqs;
  const int32_t* pages;
  const EvictPage* items;
  CacheF8 c;
  int32_t* kept;
  int64_t nkv;
  InlineMeta meta;
};
static_assert(kSmallEvict == 4 * kSelectThreads, "four keys a thread");
__global__ __launch_bounds__(kSelectThreads) void small_evict_select_kernel(SmallEvict a) {
  constexpr size_t at = offsetof(SmallEvict, meta);
  evict_select<4>(inline_meta(at, a.reqs), inline_meta(at, a.pages), a.c.weight, (int)a.nkv, a.kept);
}
template <int HD>
__global__ __launch_bounds__(256) void small_evict_move_kernel(SmallEvict a) {
  constexpr size_t at = offsetof(SmallEvict, meta);
  evict_move<HD>(inline_meta(at, a.reqs), inline_meta(at, a.pages), inline_meta(at, a.items), a.c,
                 (int)a.nkv, a.kept);
}

}  // namespace

hipError_t launch_small_append_f8(const uint16_t* k_new, const uint16_t* v_new,
                                  const CacheF8& cache, const InlineMeta& meta, int64_t n_runs,
                                  int nkv, int d, hipStream_t stream) {
  if (n_runs == 0) return hipSuccess;
  const dim3 grid((unsigned)n_runs, (2 * nkv + 3) / 4);
  const SmallAppend a{k_new, v_new, cache, nkv, meta};
  if (d == 128)
    small_append_f8_kernel<128><<<grid, 256, 0, stream>>>(a);
  else
    small_append_f8_kernel<64><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_small_evict_f8(const EvictReq* reqs, int n_reqs, const int32_t* pages,
                                 const EvictPage* items, int64_t n_items, const InlineMeta& meta,
                                 const CacheF8& cache, int32_t* kept, int nkv, int d,
                                 hipStream_t stream) {
  if (n_items == 0) return hipSuccess;
  const SmallEvict a{reqs, pages, items, cache, kept, nkv, meta};
  small_evict_select_kernel<<<dim3(n_reqs, nkv), kSelectThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)n_items, (nkv + 3) / 4);
  if (d == 128)
    small_evict_move_kernel<128><<<grid, 256, 0, stream>>>(a);
  else
    small_evict_move_kernel<64><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

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

hipError_t launch_kv_evict_f8(const EvictReq* reqs, int n_reqs, int longest, const int32_t* pages,
                              const EvictPage* items, int64_t n_items, const CacheF8& cache,
                              int32_t* kept, int nkv, int d, hipStream_t stream) {
  if (n_items == 0) return hipSuccess;
  const dim3 heads(n_reqs, nkv);
  auto select = [&](auto kernel) {
    kernel<<<heads, kSelectThreads, 0, stream>>>(reqs, pages, cache.weight, nkv, kept);
  };
  // keys a thread holds: as few as the longest request needs
  if (longest <= 4 * kSelectThreads) select(evict_select_kernel<4>);
  else if (longest <= 16 * kSelectThreads) select(evict_select_kernel<16>);
  else if (longest <= 32 * kSelectThreads) select(evict_select_kernel<32>);
  else select(evict_select_kernel<0>);
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
