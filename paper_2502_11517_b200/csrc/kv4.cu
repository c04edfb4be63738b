// The 4-bit cache: quantising append (K1 of a 4-bit pool) and read-back.  Layout of a block: device_common.cuh.
//
// 32 neighbouring elements of one token's K (or V) of one kv head are a group with a scale of its own:
//   s = the smallest number of five significant bits with amax <= 7 s over the group, kept within [2^-110, 31 * 2^106],
//   n = the whole number nearest to x / s, ties to the even one, kept within -7 ... 7; the element is held as n s.
// A token's codes depend on that token alone, so what the cache holds does not depend on how tokens were grouped into calls,
// and nothing stored is ever rounded again.  The largest element of a group comes out as n = +-7 (7 s is less than 17/16 of
// amax), so what is read back has the same scale and quantises to itself.  Five bits: n s then has at most eight significant
// bits and is a bf16 number, and s is less than 1/16 above what the group would need.
//
// An exact x / s decides a code wherever 2 x is an odd multiple of s, which for bf16 numbers is often.  Two ways, neither with
// a division per element:
//   bf16 numbers   x / s is at least 2^-10 away from k + 1/2 unless it is k + 1/2, so x (1/s) is rounded to a multiple of 2^-13
//                  first (a tie comes out as the tie it is) and to a whole number then;
//   rotated keys   (fp32) the whole number nearest to x (1/s); a lane that has a quotient within 2^-18 of the middle of two codes
//                  (one in about 10^4) compares x - n s, which is exact, with s / 2.
// An element that is not finite is stored as zero and reported (PASTA_ERR_DEVICE_CHECK), as in an 8-bit pool.
//
// One pass: 2 bytes of bf16 in and 9/16 of a byte out per element.  What bounds it: instructions (20 per element and warp in 32768 rotated
// tokens, half of them the rotation's and its exchange through shared memory), issued in 57 % of the cycles by three CTAs of eight
// warps to an SM (two, at 122 registers: 115 us with the read-back in place of 104).  Packed fp32 arithmetic does two elements per
// instruction (132 to 115 us with the checks gathered per lane).  32768 tokens: 69 us to store, 31 to read back (5.6 TB/s).
#include <cmath>
#include <type_traits>

#include "device_common.cuh"
#include "kernels.hpp"
#include "page_run.cuh"
#include "rope_form.cuh"

namespace pasta {

namespace {

constexpr float kScaleMin = 0x1p-110f, kScaleMax = 31 * 0x1p106f;

// Two fp32 numbers in a 64-bit register: one instruction for both.
using float_pair = unsigned long long;
__device__ __forceinline__ float_pair pair_of(float a, float b) {
  float_pair y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void both(float_pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ float_pair fma_pair(float_pair a, float_pair b, float_pair c) {
  float_pair y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
__device__ __forceinline__ float_pair add_pair(float_pair a, float_pair b) {
  float_pair y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ float_pair same(float a) { return pair_of(a, a); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float reciprocal(float s) {      // to an ulp
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
  return y;
}

// The scale of a group whose largest magnitude is amax (finite).  The constant is less than 1/7 by more than the product's rounding,
// so what rounding up to five bits gives is the scale or the number of five bits below it; 7 s is exact.
__device__ __forceinline__ float group_scale(float amax) {
  float s = __uint_as_float((__float_as_uint(amax * 0.14285709f) + 0x7ffffu) & 0xfff80000u);
  if (7.f * s < amax) s = __uint_as_float(__float_as_uint(s) + 0x80000u);
  return fminf(fmaxf(s, kScaleMin), kScaleMax);
}
__device__ __forceinline__ uint32_t scale_bits(float s) { return __float_as_uint(16.f * s) >> 16; }      // t, a bf16 number

constexpr float kWhole = 12582912.f;              // 1.5 * 2^23: a sum with it is a whole number
constexpr float kFine = 1536.f;                   // 1.5 * 2^10: a sum with it is a multiple of 2^-13
// whole numbers of scales nearest to two bf16 numbers, as fp32 (|x| <= 7 s); r = 1 / s
__device__ __forceinline__ float_pair codes_of_bf16(float_pair x, float_pair r) {
  return add_pair(add_pair(fma_pair(x, r, same(kFine)), same(kWhole - kFine)), same(-kWhole));
}
// the same of any fp32 number
__device__ __forceinline__ float code_of_fp32(float x, float s, float r) {
  float n = fmaf(x, r, kWhole) - kWhole;
  const float e = fmaf(-n, s, x), half = 0.5f * s;
  if (fabsf(e) >= half) {
    const bool odd = static_cast<int>(n) & 1;
    if (fabsf(e) > half || odd) n += copysignf(1.f, e);
  }
  return n;
}
// Halves of the words of eight codes n[0..7]: lo from the even ones, hi from the odd ones; two words (or both halves of one) at a time.
// The sums are whole numbers below 2^24, hence exact.
__device__ __forceinline__ float_pair code_halves(float_pair n0, float_pair n1, float_pair n2, float_pair n3) {
  return add_pair(fma_pair(n3, same(4096.f), fma_pair(n2, same(256.f), fma_pair(n1, same(16.f), n0))), same(8388608.f + 34952.f));      // 34952: 8 in each code
}
__device__ __forceinline__ uint32_t code_word(float lo, float hi) {
  const uint32_t w = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
  return __funnelshift_l(w, w, 3);
}

// 16 elements of a K row (16-element chunk c of token row r), as fp32 numbers of a bf16 row or of a rotated one; two lanes
// share a group.  amax: the largest magnitude of the 16; turned: they were rotated.  Whole warps.
template <int D, bool kRotated>
__device__ __forceinline__ void store_k16(uint8_t *block, int r, int c, bool valid, bool turned, float *x, float amax) {
  amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  const float s = group_scale(amax), inv = reciprocal(s);
  if (__any_sync(0xffffffffu, s >= kScaleMax)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = fminf(fmaxf(x[e], -7.f * s), 7.f * s);
  }
  float_pair n[8];
  if constexpr (kRotated) {
    // Rotated elements: the quotient is good to 2^-19, so the code is the nearest one unless the quotient is that close to the middle
    // of two.  The others are bf16 numbers.
    const float grid = turned ? 0.f : kFine;
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float_pair quot = fma_pair(pair_of(x[2 * i], x[2 * i + 1]), same(inv), same(grid));
      n[i] = add_pair(add_pair(quot, same(kWhole - grid)), same(-kWhole));
      float d0, d1;
      both(fma_pair(n[i], same(-1.f), quot), d0, d1);
      far = max3(far, fabsf(d0), fabsf(d1));
    }
    if (turned && far > 0.5f - 0x1p-18f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = pair_of(code_of_fp32(x[2 * i], s, inv), code_of_fp32(x[2 * i + 1], s, inv));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = codes_of_bf16(pair_of(x[2 * i], x[2 * i + 1]), same(inv));
  }
  if (!valid) return;
  float lo[2], hi[2];
  both(code_halves(n[0], n[1], n[2], n[3]), lo[0], hi[0]);
  both(code_halves(n[4], n[5], n[6], n[7]), lo[1], hi[1]);
  *reinterpret_cast<uint2 *>(block + (c >> 1) * 256 + r * 16 + (c & 1) * 8) = make_uint2(code_word(lo[0], hi[0]), code_word(lo[1], hi[1]));
  if ((c & 1) == 0)
    *reinterpret_cast<uint16_t *>(block + kv4_k_scales(D) + (r * (D / kKv4Group) + (c >> 1)) * 2) = static_cast<uint16_t>(scale_bits(s));
}

// zeros in place of numbers that are not finite; returns whether there were any
__device__ __forceinline__ bool clean_word(uint32_t &w) {
  const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
  if (lo) w &= 0xffff0000u;
  if (hi) w &= 0xffffu;
  return lo || hi;
}

// K of tokens in rows off0 .. off0 + cnt - 1 of a page, one kv head, by a warp.  rows: the tokens' K, `stride` elements apart.
// stage: this warp's room for the rotated rows of one pass (32 x 16 floats).
// The rows of a pass are asked for before those of the pass ahead of it are worked on.
template <int D, bool kRope>
__device__ __forceinline__ bool append_k(uint8_t *block, const __nv_bfloat16 *rows, int64_t stride, int off0, int cnt,
                                         const RopeForm &form, const double2 *turn, float *stage) {
  constexpr int LPT = D / 16, TPI = 32 / LPT;
  const int lane = threadIdx.x & 31, c = lane % LPT;
  const int c_a = kRope ? rope_chunk_a(form, c) : 2 * c, c_b = kRope ? rope_chunk_b(form, c) : 2 * c + 1;
  const uint4 *row = reinterpret_cast<const uint4 *>(rows + (lane / LPT) * stride);
  const int64_t step = TPI * stride / 8;
  bool bad = false;
  uint4 next_a = make_uint4(0, 0, 0, 0), next_b = next_a;
  if (lane / LPT < cnt) { next_a = __ldg(row + c_a); next_b = __ldg(row + c_b); }
#pragma unroll 1
  for (int r = lane / LPT; r - lane / LPT < cnt; r += TPI) {
    const bool valid = r < cnt;
    uint4 a = next_a, b = next_b;
    row += step;
    next_a = next_b = make_uint4(0, 0, 0, 0);
    if (r + TPI < cnt) { next_a = __ldg(row + c_a); next_b = __ldg(row + c_b); }
    const bool odd_ones = chunk_not_finite(a) || chunk_not_finite(b);
    float x[16], amax = 0.f;
    if constexpr (kRope) {
      const bool turns = c < form.slots, alternate = form.interleaved && turns;
      if (odd_ones) { bad = true; rope_clean(a, b, alternate, turns); }
      // the rotated row's chunks change hands through shared memory, so that a lane holds 16 neighbouring elements
      float *mine = stage + (lane / LPT) * D;
      auto put = [&](int chunk, const float *v) {
        float4 *dst = reinterpret_cast<float4 *>(mine + chunk * 8);
        dst[0] = make_float4(v[0], v[1], v[2], v[3]);
        dst[1] = make_float4(v[4], v[5], v[6], v[7]);
      };
      float y[16], lo[8], hi[8];
      const double2 *t = turn + (valid ? r : 0) * (D / 2);
      if (form.interleaved) {                     // (uniform: chunks stay with their lane)
        rope_slot<D>(a, b, turns, t, c, y);
        rope_unslot(y, turns, lo, hi);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] = lo[e]; x[8 + e] = hi[e]; }
      } else {
        rope_slot<D>(a, b, false, t, c, y);
        put(c_a, y);
        put(c_b, y + 8);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 v = reinterpret_cast<const float4 *>(mine + c * 16)[e];
          x[4 * e] = v.x; x[4 * e + 1] = v.y; x[4 * e + 2] = v.z; x[4 * e + 3] = v.w;
        }
        __syncwarp();
      }
#pragma unroll
      for (int e = 0; e < 16; e += 2) amax = max3(amax, fabsf(x[e]), fabsf(x[e + 1]));
      if (amax == INFINITY) {                     // a rotation that left fp32 (no NaN: its operands are finite)
        bad = true;
        amax = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] = fabsf(x[e]) == INFINITY ? 0.f : x[e];
          amax = fmaxf(amax, fabsf(x[e]));
        }
      }
    } else {
      uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      if (odd_ones) {
        bad = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) clean_word(w[i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
#pragma unroll
      for (int e = 0; e < 16; e += 2) amax = max3(amax, fabsf(x[e]), fabsf(x[e + 1]));
    }
    store_k16<D, kRope>(block, off0 + r, c, valid, kRope && c < form.slots, x, amax);
  }
  return bad;
}

// V of the same tokens, by a warp: a lane holds D / 32 channels of all 16 rows of the page.  Words (8 tokens of a channel) that
// the call does not fill are read, changed and written back; a page is worked on by one warp per call and kv head.
template <int D>
__device__ __forceinline__ bool append_v(uint8_t *block, const __nv_bfloat16 *rows, int64_t stride, int off0, int cnt) {
  constexpr int CH = D / 32, LPG = kKv4Group / CH;      // channels per lane, lanes per group
  const int lane = threadIdx.x & 31;
  bool bad = false;
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {                         // rows 8 h .. 8 h + 7: one word of every channel
    const int lo = max(off0, 8 * h), hi = min(off0 + cnt, 8 * h + 8);
    if (lo >= hi) continue;
    uint32_t x[8][CH / 2];
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 8 * h + i;
#pragma unroll
      for (int w = 0; w < CH / 2; ++w) x[i][w] = 0;
      if (r >= lo && r < hi) {
        const uint32_t *src = reinterpret_cast<const uint32_t *>(rows + (r - off0) * stride) + lane * (CH / 2);
        if constexpr (CH == 4) {
          const uint2 v = __ldg(reinterpret_cast<const uint2 *>(src));
          x[i][0] = v.x;
          x[i][1] = v.y;
        } else {
          x[i][0] = __ldg(src);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int w = 0; w < CH / 2; ++w) any = __vmaxu2(any, x[i][w] & 0x7fff7fffu);
    if ((any & 0xffffu) >= 0x7f80u || any >= 0x7f800000u) {
      bad = true;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < CH / 2; ++w) clean_word(x[i][w]);
    }
    // largest magnitudes of two tokens at a time (bf16 bits compare as integers), over the lanes of a group
    uint32_t m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t a = x[2 * j][0] & 0x7fff7fffu, b = x[2 * j + 1][0] & 0x7fff7fffu;
      if constexpr (CH == 4) {
        a = __vmaxu2(a, x[2 * j][1] & 0x7fff7fffu);
        b = __vmaxu2(b, x[2 * j + 1][1] & 0x7fff7fffu);
      }
      m[j] = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
      for (int o = 1; o < LPG; o <<= 1) m[j] = __vmaxu2(m[j], __shfl_xor_sync(0xffffffffu, m[j], o));
    }
    // lane i of a group works out the scale of token i, and keeps it; the others ask for 1 / s
    const int who = lane & 7;
    const uint32_t pair = (who & 4) ? ((who & 2) ? m[3] : m[2]) : ((who & 2) ? m[1] : m[0]);
    const float s = group_scale((who & 1) ? bf16_hi(pair) : bf16_lo(pair)), inv = reciprocal(s);
    if ((lane & (LPG - 1)) < 8 && 8 * h + who >= lo && 8 * h + who < hi)
      *reinterpret_cast<uint16_t *>(block + kv4_v_scales(D) + (lane / LPG) * 32 + (8 * h + who) * 2) = static_cast<uint16_t>(scale_bits(s));
    float_pair n[CH / 2][8];                            // of two neighbouring channels
    auto codes = [&](auto clamp) {                      // clamp: some elements may be beyond 7 scales
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float r = __shfl_sync(0xffffffffu, inv, (lane & ~7) | i);
        const float most = decltype(clamp)::value ? 7.f * __shfl_sync(0xffffffffu, s, (lane & ~7) | i) : 0.f;
#pragma unroll
        for (int w = 0; w < CH / 2; ++w) {
          float v0 = bf16_lo(x[i][w]), v1 = bf16_hi(x[i][w]);
          if (decltype(clamp)::value) { v0 = fminf(fmaxf(v0, -most), most); v1 = fminf(fmaxf(v1, -most), most); }
          n[w][i] = codes_of_bf16(pair_of(v0, v1), same(r));
        }
      }
    };
    if (__any_sync(0xffffffffu, s >= kScaleMax)) codes(std::true_type());
    else codes(std::false_type());
    uint32_t *dst = reinterpret_cast<uint32_t *>(block + kv4_v_codes(D)) + lane * CH * 2 + h;
    uint32_t keep = 0;                                  // bits of the word that hold other tokens
    if (hi - lo < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * h + i < lo || 8 * h + i >= hi) keep |= 0xfu << ((i & 1) * 16 + (i >> 1) * 4);
      keep = __funnelshift_l(keep, keep, 3);
    }
#pragma unroll
    for (int w = 0; w < CH / 2; ++w) {
      float lo[2], hi[2];
      both(code_halves(n[w][0], n[w][2], n[w][4], n[w][6]), lo[0], lo[1]);
      both(code_halves(n[w][1], n[w][3], n[w][5], n[w][7]), hi[0], hi[1]);
#pragma unroll
      for (int ch = 2 * w; ch < 2 * w + 2; ++ch) {
        uint32_t word = code_word(lo[ch & 1], hi[ch & 1]);
        if (keep) word = (word & ~keep) | (dst[2 * ch] & keep);
        dst[2 * ch] = word;
      }
    }
  }
  return bad;
}

template <int D, bool kRope>
struct AppendSmem {
  double2 turn[kRope ? PASTA_PAGE * (D / 2) : 1];
  float stage[kRope ? A_WARPS : 1][kRope ? 512 : 4];
};

// The new tokens that fall into one page, layers ll .. ll_end - 1, by one CTA: a warp takes one (kv head, K or V) at a time.
template <int D, bool kRope>
__device__ __forceinline__ void append_page4(const PoolView &pv, int page, int off0, int first, int cnt, int layer_begin, int ll, int ll_end,
                                             int64_t in_layer_stride, const __nv_bfloat16 *__restrict__ k_new,
                                             const __nv_bfloat16 *__restrict__ v_new, const RopeForm &form, AppendSmem<D, kRope> &sm) {
  const int warp = threadIdx.x >> 5;
  const int H = pv.n_kv_heads;
  const int64_t stride = static_cast<int64_t>(H) * D;
  for (; ll < ll_end; ++ll) {
    if (ll + 1 < ll_end) prefetch_rows(k_new, v_new, (ll + 1) * in_layer_stride + first * stride, cnt * H * D * 2);
    uint8_t *layer = pv.kv_base + (layer_begin + ll) * pv.layer_stride;
    for (int item = warp; item < 2 * H; item += A_WARPS) {
      const int g = item >> 1, kv = (item ^ (item / A_WARPS)) & 1;      // a warp's items are K and V in turn
      uint8_t *block = layer + (static_cast<int64_t>(page) * H + g) * kv4_block_bytes(D);
      const int64_t at = ll * in_layer_stride + first * stride + g * D;
      const bool bad = kv ? append_v<D>(block, v_new + at, stride, off0, cnt)
                          : append_k<D, kRope>(block, k_new + at, stride, off0, cnt, form, sm.turn, sm.stage[kRope ? warp : 0]);
      if (bad) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    }
  }
}

// Tokens of a step: slots[2 i], slots[2 i + 1] are token i's page and row.  One CTA per group of tokens that are neighbours in
// one page (the CTA of a group's first token takes it) and slice of the layers.
template <int D, bool kRope>
__global__ void __launch_bounds__(A_THREADS, 3)
kv4_append_kernel(PoolView pv, const int32_t *__restrict__ slots, const int32_t *__restrict__ pos, int32_t n_tok,
                  int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta, int64_t in_layer_stride,
                  const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new, const __grid_constant__ RopeForm form) {
  __shared__ AppendSmem<D, kRope> sm;
  grid_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31;
  const int first = blockIdx.x;
  const int page = slots[2 * first], off0 = slots[2 * first + 1];
  if (first > 0 && slots[2 * first - 2] == page && slots[2 * first - 1] == off0 - 1) return;
  const int a = first + lane;
  const bool mine = lane < PASTA_PAGE && a < n_tok && slots[2 * a] == page && slots[2 * a + 1] == off0 + lane;
  const int cnt = __ffs(~__ballot_sync(0xffffffffu, mine)) - 1;
  if (page < 0 || page >= pv.n_pages || off0 < 0 || off0 + cnt > PASTA_PAGE || cnt < 1) {
    if (tid == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  if constexpr (kRope) {
    for (int x = tid; x < cnt * (D / 2); x += A_THREADS)
      sm.turn[x / (D / 2) * (D / 2) + turn_at<D>(x % (D / 2))] = turn_of(form, x % (D / 2), pos[first + x / (D / 2)]);
    __syncthreads();
  }
  const int ll = blockIdx.y * layers_per_cta;
  append_page4<D, kRope>(pv, page, off0, first, cnt, layer_begin, ll, min(layer_count, ll + layers_per_cta), in_layer_stride, k_new, v_new, form, sm);
}

// A run: n_tok tokens of one stream at consecutive positions, the first at row first_offset of the first page.  One CTA per
// page and slice of the layers.
template <int D, bool kRope, int N>
__global__ void __launch_bounds__(A_THREADS, 3)
kv4_append_run_kernel(PoolView pv, const __grid_constant__ PageList<N> pages, int32_t pos0, int32_t n_tok, int32_t first_offset,
                      int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta, int64_t in_layer_stride,
                      const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new, const __grid_constant__ RopeForm form) {
  __shared__ AppendSmem<D, kRope> sm;
  grid_launch_dependents();
  const int first = max(0, static_cast<int>(blockIdx.x) * PASTA_PAGE - first_offset);
  const int cnt = min(n_tok, (static_cast<int>(blockIdx.x) + 1) * PASTA_PAGE - first_offset) - first;
  const int page = pages.page[blockIdx.x], off0 = blockIdx.x == 0 ? first_offset : 0;
  if (page < 0 || page >= pv.n_pages || cnt < 1) {
    if (threadIdx.x == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  const int ll = blockIdx.y * layers_per_cta;
  prefetch_rows(k_new, v_new, ll * in_layer_stride + static_cast<int64_t>(first) * pv.n_kv_heads * D, cnt * pv.n_kv_heads * D * 2);
  if constexpr (kRope) {
    turns_of_run<D, A_THREADS>(form, pos0 + first, cnt, sm.turn);
    __syncthreads();
  }
  append_page4<D, kRope>(pv, page, off0, first, cnt, layer_begin, ll, min(layer_count, ll + layers_per_cta), in_layer_stride, k_new, v_new, form, sm);
}

// A run read back: one CTA per page and layer (blockIdx.y), a warp per (kv head, K or V).
template <int D, int N>
__global__ void __launch_bounds__(A_THREADS, 4)
kv4_read_kernel(PoolView pv, const __grid_constant__ PageList<N> pages, int32_t n_tok, int32_t first_offset, int32_t layer_begin,
                int64_t out_layer_stride, __nv_bfloat16 *__restrict__ k_out, __nv_bfloat16 *__restrict__ v_out) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = static_cast<int>(blockIdx.x) * PASTA_PAGE - first_offset;       // token of the page's first row
  const int page = pages.page[blockIdx.x];
  if (page < 0 || page >= pv.n_pages) {
    if (threadIdx.x == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  const int H = pv.n_kv_heads;
  const uint8_t *layer = pv.kv_base + (layer_begin + static_cast<int64_t>(blockIdx.y)) * pv.layer_stride;
  for (int item = warp; item < 2 * H; item += A_WARPS) {
    const int g = item >> 1;
    const uint8_t *block = layer + (static_cast<int64_t>(page) * H + g) * kv4_block_bytes(D);
    if ((item & 1) == 0) {                            // K: a lane turns 16 codes of a row into 32 bytes
      constexpr int LPT = D / 16, TPI = 32 / LPT, NI = PASTA_PAGE / TPI;
      const int c = lane % LPT;
      uint2 q[NI];
      uint32_t t[NI];
#pragma unroll
      for (int it = 0; it < NI; ++it) {
        const int r = it * TPI + lane / LPT;
        q[it] = *reinterpret_cast<const uint2 *>(block + (c >> 1) * 256 + r * 16 + (c & 1) * 8);
        t[it] = *reinterpret_cast<const uint16_t *>(block + kv4_k_scales(D) + (r * (D / kKv4Group) + (c >> 1)) * 2);
      }
#pragma unroll
      for (int it = 0; it < NI; ++it) {
        const int tok = first + it * TPI + lane / LPT;
        if (tok < 0 || tok >= n_tok) continue;
        const uint32_t t2 = t[it] | (t[it] << 16), c2 = kv4_offset_of(t2);
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[i] = kv4_value(kv4_pair(q[it].x, i), t2, c2);
          o[4 + i] = kv4_value(kv4_pair(q[it].y, i), t2, c2);
        }
        uint4 *dst = reinterpret_cast<uint4 *>(k_out + blockIdx.y * out_layer_stride + (static_cast<int64_t>(tok) * H + g) * D + c * 16);
        dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
        dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    } else {                                          // V: a lane turns D / 32 channels of 16 tokens
      constexpr int CH = D / 32, LPG = kKv4Group / CH;
      uint32_t w[CH][2], t[8];
#pragma unroll
      for (int ch = 0; ch < CH; ch += 2) {
        const uint4 v = *reinterpret_cast<const uint4 *>(block + kv4_v_codes(D) + (lane * CH + ch) * 8);
        w[ch][0] = v.x; w[ch][1] = v.y; w[ch + 1][0] = v.z; w[ch + 1][1] = v.w;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 v = *reinterpret_cast<const uint4 *>(block + kv4_v_scales(D) + (lane / LPG) * 32 + j * 16);
        t[4 * j] = v.x; t[4 * j + 1] = v.y; t[4 * j + 2] = v.z; t[4 * j + 3] = v.w;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {                   // tokens 2 j and 2 j + 1
        const uint32_t c2 = kv4_offset_of(t[j]);
        uint32_t v[CH];
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) v[ch] = kv4_value(kv4_pair(w[ch][j >> 2], j & 3), t[j], c2);
#pragma unroll
        for (int up = 0; up < 2; ++up) {
          const int tok = first + 2 * j + up;
          if (tok < 0 || tok >= n_tok) continue;
          uint32_t *dst = reinterpret_cast<uint32_t *>(v_out + blockIdx.y * out_layer_stride + (static_cast<int64_t>(tok) * H + g) * D) + lane * (CH / 2);
          if constexpr (CH == 4)
            *reinterpret_cast<uint2 *>(dst) = make_uint2(__byte_perm(v[0], v[1], up ? 0x7632 : 0x5410), __byte_perm(v[2], v[3], up ? 0x7632 : 0x5410));
          else
            *dst = __byte_perm(v[0], v[1], up ? 0x7632 : 0x5410);
        }
      }
    }
  }
}

template <int N>
cudaError_t launch_append_pages(const PoolView &pv, const int32_t *pages, int n_pages, int32_t pos0, int32_t n_tok, int32_t first_offset,
                                int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const __nv_bfloat16 *k,
                                const __nv_bfloat16 *v, const RopeForm *form, cudaStream_t st) {
  static const RopeForm none{};
  const PageList<N> list = list_of<N>(pages, n_pages);
  const int per = layers_per_cta(n_pages, layer_count);
  const dim3 grid(n_pages, (layer_count + per - 1) / per);
  const auto kernel = pv.head_dim == 128 ? (form ? kv4_append_run_kernel<128, true, N> : kv4_append_run_kernel<128, false, N>)
                                         : (form ? kv4_append_run_kernel<64, true, N> : kv4_append_run_kernel<64, false, N>);
  kernel<<<grid, A_THREADS, 0, st>>>(pv, list, pos0, n_tok, first_offset, layer_begin, layer_count, per, in_layer_stride, k, v,
                                     form ? *form : none);
  return cudaGetLastError();
}

template <int N>
cudaError_t launch_read_pages(const PoolView &pv, const int32_t *pages, int n_pages, int32_t n_tok, int32_t first_offset,
                              int32_t layer_begin, int32_t layer_count, int64_t out_layer_stride, __nv_bfloat16 *k, __nv_bfloat16 *v,
                              cudaStream_t st) {
  const PageList<N> list = list_of<N>(pages, n_pages);
  const auto kernel = pv.head_dim == 128 ? kv4_read_kernel<128, N> : kv4_read_kernel<64, N>;
  kernel<<<dim3(n_pages, layer_count), A_THREADS, 0, st>>>(pv, list, n_tok, first_offset, layer_begin, out_layer_stride, k, v);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_append(const PoolView &pv, const int32_t *slots, const int32_t *pos, int32_t n_tok, int32_t layer_begin,
                              int32_t layer_count, int64_t in_layer_stride, const void *k_new, const void *v_new,
                              const RopeForm *form, cudaStream_t st) {
  if (n_tok == 0 || layer_count == 0) return cudaSuccess;
  static const RopeForm none{};
  const int per = layers_per_cta(n_tok, layer_count);
  const dim3 grid(n_tok, (layer_count + per - 1) / per);
  const auto kernel = pv.head_dim == 128 ? (form ? kv4_append_kernel<128, true> : kv4_append_kernel<128, false>)
                                         : (form ? kv4_append_kernel<64, true> : kv4_append_kernel<64, false>);
  kernel<<<grid, A_THREADS, 0, st>>>(pv, slots, pos, n_tok, layer_begin, layer_count, per, in_layer_stride,
                                     static_cast<const __nv_bfloat16 *>(k_new), static_cast<const __nv_bfloat16 *>(v_new), form ? *form : none);
  return cudaGetLastError();
}

cudaError_t launch_kv4_append_run(const PoolView &pv, const int32_t *pages, int32_t first_offset, int32_t pos0, int32_t n_tok,
                                  int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const void *k_new,
                                  const void *v_new, const RopeForm *form, cudaStream_t st, int64_t *launches) {
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(k_new), *v = static_cast<const __nv_bfloat16 *>(v_new);
  const int64_t tok = static_cast<int64_t>(pv.n_kv_heads) * pv.head_dim;
  for (int32_t done = 0; done < n_tok;) {
    const int32_t left = n_tok - done, all = (first_offset + left + PASTA_PAGE - 1) / PASTA_PAGE;
    const int32_t n = std::min(all, kPagesLarge), cnt = std::min(left, n * PASTA_PAGE - first_offset);
    const auto launch = n <= kPagesSmall ? launch_append_pages<kPagesSmall> : launch_append_pages<kPagesLarge>;
    const cudaError_t e = launch(pv, pages, n, pos0 + done, cnt, first_offset, layer_begin, layer_count, in_layer_stride, k + done * tok,
                                 v + done * tok, form, st);
    if (e != cudaSuccess) return e;
    *launches += 1;
    pages += n;
    done += cnt;
    first_offset = 0;
  }
  return cudaSuccess;
}

cudaError_t launch_kv4_read_run(const PoolView &pv, const int32_t *pages, int32_t first_offset, int32_t n_tok, int32_t layer_begin,
                                int32_t layer_count, int64_t out_layer_stride, void *k_out, void *v_out, cudaStream_t st,
                                int64_t *launches) {
  __nv_bfloat16 *k = static_cast<__nv_bfloat16 *>(k_out), *v = static_cast<__nv_bfloat16 *>(v_out);
  const int64_t tok = static_cast<int64_t>(pv.n_kv_heads) * pv.head_dim;
  for (int32_t done = 0; done < n_tok;) {
    const int32_t left = n_tok - done, all = (first_offset + left + PASTA_PAGE - 1) / PASTA_PAGE;
    const int32_t n = std::min(all, kPagesLarge), cnt = std::min(left, n * PASTA_PAGE - first_offset);
    const auto launch = n <= kPagesSmall ? launch_read_pages<kPagesSmall> : launch_read_pages<kPagesLarge>;
    const cudaError_t e = launch(pv, pages, n, cnt, first_offset, layer_begin, layer_count, out_layer_stride, k + done * tok, v + done * tok, st);
    if (e != cudaSuccess) return e;
    *launches += 1;
    pages += n;
    done += cnt;
    first_offset = 0;
  }
  return cudaSuccess;
}

}  // namespace pasta
