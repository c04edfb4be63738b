// The 8-bit cache: quantising append (K1 of an 8-bit pool) and read-back.
//
// A page (16 tokens of one stream) has, per layer and kv head, one scale for K and one for V, a power of two 2^e:
//   e = the smallest integer with amax <= 448 * 2^e over the page's elements, kept within [-64, 63] (a page of zeros: -64),
//   code = e4m3 nearest to x * 2^-e, ties to even, magnitudes above 448 held at 448.
// e4m3 is a floating-point format, so a power-of-two scale loses nothing against a finer one except at the very bottom of
// the range, and it makes a scale's growth exact: tokens arrive one at a time, and when a later one needs a larger e the
// codes already in the page are multiplied by 2^-(growth), which changes no code except those that become subnormal
// (below 2^-6 of the new scale: one more rounding, at most half a step of the new scale).  e never shrinks while a page
// fills and starts anew with the page's first slot.
// An element that is not finite is stored as zero and reported (PASTA_ERR_DEVICE_CHECK): a cache that holds only finite
// values cannot spoil rows that do not see the token.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "device_common.cuh"
#include "kernels.hpp"

namespace pasta {

namespace {

constexpr int A_THREADS = 256, A_WARPS = A_THREADS / 32;

// Rotation by angle i = f[i] times the position, f[i] = theta^(-2i/D); (c1[i], s1[i]) is the rotation by one position.
struct Freqs { double f[64], c1[64], s1[64]; };
// The pages of a run, as kernel arguments (a run needs no copy to the device before it); two sizes, since every launch
// carries the whole array.
template <int N> struct PageList { int32_t page[N]; };
constexpr int kPagesSmall = 64, kPagesLarge = 2048;

// Sines and cosines are kept times 2^896, and a bf16 number becomes the 64-bit number whose exponent field is its own: that
// is the number times 2^-896, subnormal or not, for two integer instructions in place of a conversion (measured: 17 cycles
// per warp for a conversion there and back, 2 for a multiplication).  Infinities and NaN are sorted out before.
constexpr double kTurnScale = 0x1p896;
__device__ __forceinline__ double scaled_down(uint32_t bits) {       // bits: fp32 bits of a bf16 number
  return __hiloint2double((static_cast<int>(bits) >> 3) & 0x8fffffff, 0);
}

// exponent of the scale for a largest magnitude given by its fp32 bits (finite)
__device__ __forceinline__ int scale_exp(uint32_t amax_bits) {
  const int e = static_cast<int>(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
  return min(max(e, kKv8ExpMin), kKv8ExpMax);
}

// The scale of one (page, kv head, K or V) after tokens with the given amax join rows [0, off0): grows the scale and moves
// the codes already there when needed.  Whole warp; returns the exponent.
template <int D>
__device__ __forceinline__ int grow_scale(uint8_t *block, int8_t *scale, int kv, int off0, uint32_t amax_bits, int lane) {
  int e = scale_exp(amax_bits);
  if (off0 > 0) {
    const int old = *scale;
    if (e > old) {
      const float f = pow2f(max(old - e, -126));
      for (int w = lane; w < off0 * (D / 4); w += 32) {
        const int r = w / (D / 4), x = w % (D / 4);
        uint32_t *at = reinterpret_cast<uint32_t *>(block + ((r >> 3) * 2 + kv) * (8 * D) + (r & 7) * D) + x;
        uint32_t lo, hi;
        e4m3x4_to_f16x4(*at, lo, hi);
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo)), b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
        *at = e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
      }
    } else {
      e = old;
    }
  }
  __syncwarp();
  if (lane == 0) *scale = static_cast<int8_t>(e);
  return e;
}

// Rows of one layer on their way into L2 while the CTA works on something else (16-byte aligned, as the loads require).
__device__ __forceinline__ void prefetch_rows(const __nv_bfloat16 *k_new, const __nv_bfloat16 *v_new, int64_t at, int bytes) {
  if (threadIdx.x < 2)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"((threadIdx.x ? v_new : k_new) + at), "r"(bytes) : "memory");
}

// The new tokens that fall into one page (rows off0 .. off0 + cnt - 1 of it), layers ll .. ll_end - 1, by one CTA: a warp takes
// one (kv head, K or V) at a time, holds the group's elements in registers, finds their largest magnitude, and writes the
// codes, so every element is read once.  turn: (cos, sin) of token r, angle i = 8 c + e at r * H + e * (H / 8) + c.
template <int D, bool kRope>
__device__ __forceinline__ void append_page(const PoolView &pv, int page, int off0, int first, int cnt, int layer_begin, int ll, int ll_end,
                                            int64_t in_layer_stride, const __nv_bfloat16 *__restrict__ k_new,
                                            const __nv_bfloat16 *__restrict__ v_new, const double2 *turn) {
  constexpr int H = D / 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int Hkv = pv.n_kv_heads;
  for (; ll < ll_end; ++ll) {
    if (ll + 1 < ll_end) prefetch_rows(k_new, v_new, (ll + 1) * in_layer_stride + static_cast<int64_t>(first) * Hkv * D, cnt * Hkv * D * 2);
    uint8_t *layer = pv.kv_base + (layer_begin + ll) * pv.layer_stride;
    for (int item = warp; item < 2 * Hkv; item += A_WARPS) {
      const int g = item >> 1, kv = (item ^ (item / A_WARPS)) & 1;      // a warp's items are K and V in turn
      const __nv_bfloat16 *src = (kv ? v_new : k_new) + ll * in_layer_stride + (static_cast<int64_t>(first) * Hkv + g) * D;
      const int64_t at = static_cast<int64_t>(page) * Hkv + g;
      uint8_t *block = layer + at * kv8_block_bytes(D);
      int8_t *scale = reinterpret_cast<int8_t *>(layer + pv.scale_off) + at * 2 + kv;
      bool bad = false;
      if (kRope && kv == 0) {
        // a lane holds the 8 elements of chunk c of the low half and the 8 they pair with in the high half
        constexpr int LPT = D / 16, TPI = 32 / LPT, NI = PASTA_PAGE / TPI;
        const int c = lane % LPT;
        float y[NI][16], top = 0.f;
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const int r = it * TPI + lane / LPT;
          if (r < cnt) {
            const uint4 *row = reinterpret_cast<const uint4 *>(src + static_cast<int64_t>(r) * Hkv * D);
            const uint4 lo4 = __ldg(row + c), hi4 = __ldg(row + c + LPT);
            uint32_t lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
            uint32_t m2 = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) m2 = __vmaxu2(m2, __vmaxu2(lo[w] & 0x7fff7fffu, hi[w] & 0x7fff7fffu));
            if ((m2 & 0xffffu) >= 0x7f80u || m2 >= 0x7f800000u) {     // a pair with a number that is not finite: both are zeros
              bad = true;
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const uint32_t x2 = __vmaxu2(lo[w] & 0x7fff7fffu, hi[w] & 0x7fff7fffu);
                const uint32_t keep = ((x2 & 0xffffu) >= 0x7f80u ? 0u : 0xffffu) | (x2 >= 0x7f800000u ? 0u : 0xffff0000u);
                lo[w] &= keep;
                hi[w] &= keep;
              }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const double2 t = turn[r * H + e * (H / 8) + c];
              const double a = scaled_down((e & 1) ? lo[e >> 1] & 0xffff0000u : lo[e >> 1] << 16);
              const double b = scaled_down((e & 1) ? hi[e >> 1] & 0xffff0000u : hi[e >> 1] << 16);
              y[it][e] = static_cast<float>(a * t.x - b * t.y);
              y[it][8 + e] = static_cast<float>(b * t.x + a * t.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[it][e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(y[it][e]));
        }
        if (__any_sync(0xffffffffu, top == INFINITY)) {           // a rotation that left fp32 (no NaN: its operands are finite)
          top = 0.f;
#pragma unroll
          for (int it = 0; it < NI; ++it)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if (fabsf(y[it][e]) == INFINITY) { y[it][e] = 0.f; bad = true; }
              top = fmaxf(top, fabsf(y[it][e]));
            }
        }
        const uint32_t amax = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
        const float inv = pow2f(-grow_scale<D>(block, scale, 0, off0, amax, lane));
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const int r = it * TPI + lane / LPT;
          if (r < cnt) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float *z = y[it] + 8 * half;
              const int c8 = c + half * LPT;            // 8-element chunk of the row
              *reinterpret_cast<uint2 *>(block + kv8_chunk_offset<D>(0, off0 + r, c8 >> 1) + (c8 & 1) * 8) =
                  make_uint2(e4m3x4(z[0] * inv, z[1] * inv, z[2] * inv, z[3] * inv),
                             e4m3x4(z[4] * inv, z[5] * inv, z[6] * inv, z[7] * inv));
            }
          }
        }
      } else {
        constexpr int LPT = D / 8, TPI = 32 / LPT, NI = PASTA_PAGE / TPI;
        const int c = lane % LPT;
        uint32_t x[NI][4];
        uint32_t amax2 = 0;                  // two 16-bit maxima of magnitudes
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const int r = it * TPI + lane / LPT;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (r < cnt) v = __ldg(reinterpret_cast<const uint4 *>(src + static_cast<int64_t>(r) * Hkv * D) + c);
          x[it][0] = v.x; x[it][1] = v.y; x[it][2] = v.z; x[it][3] = v.w;
        }
#pragma unroll
        for (int it = 0; it < NI; ++it)
#pragma unroll
          for (int w = 0; w < 4; ++w) amax2 = __vmaxu2(amax2, x[it][w] & 0x7fff7fffu);
        if (__any_sync(0xffffffffu, (amax2 & 0xffffu) >= 0x7f80u || (amax2 >> 16) >= 0x7f80u)) {
          amax2 = 0;
#pragma unroll
          for (int it = 0; it < NI; ++it)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if ((x[it][w] & 0x7f80u) == 0x7f80u) { x[it][w] &= 0xffff0000u; bad = true; }
              if ((x[it][w] & 0x7f800000u) == 0x7f800000u) { x[it][w] &= 0xffffu; bad = true; }
              amax2 = __vmaxu2(amax2, x[it][w] & 0x7fff7fffu);
            }
        }
        const uint32_t amax = __reduce_max_sync(0xffffffffu, max(amax2 << 16, amax2 & 0xffff0000u));
        const float inv = pow2f(-grow_scale<D>(block, scale, kv, off0, amax, lane));
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const int r = it * TPI + lane / LPT;
          if (r < cnt)
            *reinterpret_cast<uint2 *>(block + kv8_chunk_offset<D>(kv, off0 + r, c >> 1) + (c & 1) * 8) =
                make_uint2(e4m3x4(bf16_lo(x[it][0]) * inv, bf16_hi(x[it][0]) * inv, bf16_lo(x[it][1]) * inv, bf16_hi(x[it][1]) * inv),
                           e4m3x4(bf16_lo(x[it][2]) * inv, bf16_hi(x[it][2]) * inv, bf16_lo(x[it][3]) * inv, bf16_hi(x[it][3]) * inv));
        }
      }
      if (bad) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    }
  }
}

// Tokens of a step: slots[2 i], slots[2 i + 1] are token i's page and row.  One CTA per group of tokens that are neighbours in
// one page (the CTA of a group's first token takes it) and slice of the layers; the sines and cosines (64 bits) are worked
// out once per CTA for all heads and layers.
template <int D, bool kRope>
__global__ void __launch_bounds__(A_THREADS, kRope ? 2 : 3)
kv8_append_kernel(PoolView pv, const int32_t *__restrict__ slots, const int32_t *__restrict__ pos, int32_t n_tok,
                  int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta, int64_t in_layer_stride,
                  const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new, const __grid_constant__ Freqs freqs) {
  constexpr int H = D / 2;
  __shared__ double2 turn[kRope ? PASTA_PAGE * H : 1];
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
  if (kRope) {
    for (int x = tid; x < cnt * H; x += A_THREADS) {
      const int r = x / H, i = x % H;
      double sn, cs;
      sincos(static_cast<double>(pos[first + r]) * freqs.f[i], &sn, &cs);
      turn[r * H + (i & 7) * (H / 8) + (i >> 3)] = make_double2(cs * kTurnScale, sn * kTurnScale);
    }
    __syncthreads();
  }
  const int ll = blockIdx.y * layers_per_cta;
  append_page<D, kRope>(pv, page, off0, first, cnt, layer_begin, ll, min(layer_count, ll + layers_per_cta), in_layer_stride, k_new, v_new, turn);
}

// A run: n_tok tokens of one stream at consecutive positions, the first at row first_offset of the first page.  One CTA per
// page and slice of the layers.  A thread works out the sine and cosine of one angle at every fourth token and turns it on by
// one position at a time for the three behind it: three products, each good to a few times 2^-53.
template <int D, bool kRope, int N>
__global__ void __launch_bounds__(A_THREADS, kRope ? 2 : 3)
kv8_append_run_kernel(PoolView pv, const __grid_constant__ PageList<N> pages, int32_t pos0, int32_t n_tok, int32_t first_offset,
                      int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta, int64_t in_layer_stride,
                      const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new, const __grid_constant__ Freqs freqs) {
  constexpr int H = D / 2;
  __shared__ double2 turn[kRope ? PASTA_PAGE * H : 1];
  grid_launch_dependents();
  const int tid = threadIdx.x;
  const int first = max(0, static_cast<int>(blockIdx.x) * PASTA_PAGE - first_offset);
  const int cnt = min(n_tok, (static_cast<int>(blockIdx.x) + 1) * PASTA_PAGE - first_offset) - first;
  const int page = pages.page[blockIdx.x], off0 = blockIdx.x == 0 ? first_offset : 0;
  if (page < 0 || page >= pv.n_pages || cnt < 1) {
    if (tid == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  const int ll = blockIdx.y * layers_per_cta;
  prefetch_rows(k_new, v_new, ll * in_layer_stride + static_cast<int64_t>(first) * pv.n_kv_heads * D, cnt * pv.n_kv_heads * D * 2);
  if (kRope) {
    for (int x = tid; x < PASTA_PAGE / 4 * H; x += A_THREADS) {
      const int r = x / H * 4, i = x % H;
      double2 *at = turn + r * H + (i & 7) * (H / 8) + (i >> 3);
      double sn = 0, cs = 0;
      if (r < cnt) sincos(static_cast<double>(pos0 + first + r) * freqs.f[i], &sn, &cs);
      cs *= kTurnScale;
      sn *= kTurnScale;
      const double c1 = freqs.c1[i], s1 = freqs.s1[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (r + j < cnt) at[j * H] = make_double2(cs, sn);
        const double next = cs * c1 - sn * s1;
        sn = sn * c1 + cs * s1;
        cs = next;
      }
    }
    __syncthreads();
  }
  append_page<D, kRope>(pv, page, off0, first, cnt, layer_begin, ll, min(layer_count, ll + layers_per_cta), in_layer_stride, k_new, v_new, turn);
}

// A run read back: one CTA per page and layer (blockIdx.y), a warp per (kv head, K or V); a lane turns 16 codes into 32 bytes.
template <int D, int N>
__global__ void __launch_bounds__(A_THREADS, 4)
kv8_read_kernel(PoolView pv, const __grid_constant__ PageList<N> pages, int32_t n_tok, int32_t first_offset, int32_t layer_begin,
                int64_t out_layer_stride, __nv_bfloat16 *__restrict__ k_out, __nv_bfloat16 *__restrict__ v_out) {
  constexpr int LPT = D / 16, TPI = 32 / LPT, NI = PASTA_PAGE / TPI;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane % LPT;
  const int first = static_cast<int>(blockIdx.x) * PASTA_PAGE - first_offset;       // token of the page's first row
  const int page = pages.page[blockIdx.x];
  if (page < 0 || page >= pv.n_pages) {
    if (threadIdx.x == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  const int Hkv = pv.n_kv_heads;
  const uint8_t *layer = pv.kv_base + (layer_begin + static_cast<int64_t>(blockIdx.y)) * pv.layer_stride;
  for (int item = warp; item < 2 * Hkv; item += A_WARPS) {
    const int g = item >> 1, kv = item & 1;
    const int64_t at = static_cast<int64_t>(page) * Hkv + g;
    const uint8_t *block = layer + at * kv8_block_bytes(D);
    const int ex = *(reinterpret_cast<const int8_t *>(layer + pv.scale_off) + at * 2 + kv);
    __nv_bfloat16 *out = (kv ? v_out : k_out) + blockIdx.y * out_layer_stride + g * D + c * 16;
    uint4 q[NI];
#pragma unroll
    for (int it = 0; it < NI; ++it)
      q[it] = *reinterpret_cast<const uint4 *>(block + kv8_chunk_offset<D>(kv, it * TPI + lane / LPT, c));
    const float f = pow2f(ex);
#pragma unroll
    for (int it = 0; it < NI; ++it) {
      const int t = first + it * TPI + lane / LPT;
      if (t < 0 || t >= n_tok) continue;
      const uint32_t w[4] = {q[it].x, q[it].y, q[it].z, q[it].w};
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t h[2];
        e4m3x4_to_f16x4(w[i], h[0], h[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h[j]));
          const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * f, v.y * f);          // exact: four significant bits
          o[2 * i + j] = *reinterpret_cast<const uint32_t *>(&b);
        }
      }
      uint4 *dst = reinterpret_cast<uint4 *>(out + static_cast<int64_t>(t) * Hkv * D);
      dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
      dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
  }
}

// the frequencies of a theta, worked out again only when it changes (one table per host thread)
const Freqs &freqs_of(double theta, int head_dim) {
  static thread_local Freqs fr;
  static thread_local double of = 0;
  static thread_local int dim = 0;
  if (of != theta || dim != head_dim) {
    for (int i = 0; i < head_dim / 2; ++i) {
      fr.f[i] = std::exp2(-2.0 * i / head_dim * std::log2(theta));
      fr.c1[i] = std::cos(fr.f[i]);
      fr.s1[i] = std::sin(fr.f[i]);
    }
    of = theta;
    dim = head_dim;
  }
  return fr;
}

// layers per CTA: all layers of a page in one CTA share its sines and cosines; split only as far as the GPU has to be filled
int layers_per_cta(int groups, int layer_count) {
  const int want = 148 * 2;          // (twice as many: 35.4 against 33.3 us for 64 pages of 8 layers with rotation)
  const int slices = std::min(layer_count, std::max(1, (want + groups - 1) / groups));
  return (layer_count + slices - 1) / slices;
}

template <int N>
PageList<N> list_of(const int32_t *pages, int n) {
  PageList<N> list;
  std::copy(pages, pages + n, list.page);
  return list;
}

template <int N>
cudaError_t launch_append_pages(const PoolView &pv, const int32_t *pages, int n_pages, int32_t pos0, int32_t n_tok, int32_t first_offset,
                                int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const __nv_bfloat16 *k,
                                const __nv_bfloat16 *v, double theta, cudaStream_t st) {
  const PageList<N> list = list_of<N>(pages, n_pages);
  const int per = layers_per_cta(n_pages, layer_count);
  const dim3 grid(n_pages, (layer_count + per - 1) / per);
  const Freqs &fr = freqs_of(theta > 0 ? theta : 2.0, pv.head_dim);
#define PASTA_A8(DD, RR)                                                                                                \
  kv8_append_run_kernel<DD, RR, N><<<grid, A_THREADS, 0, st>>>(pv, list, pos0, n_tok, first_offset, layer_begin, layer_count, per, \
                                                               in_layer_stride, k, v, fr)
  if (pv.head_dim == 128) { if (theta > 0) PASTA_A8(128, true); else PASTA_A8(128, false); }
  else { if (theta > 0) PASTA_A8(64, true); else PASTA_A8(64, false); }
#undef PASTA_A8
  return cudaGetLastError();
}

template <int N>
cudaError_t launch_read_pages(const PoolView &pv, const int32_t *pages, int n_pages, int32_t n_tok, int32_t first_offset,
                              int32_t layer_begin, int32_t layer_count, int64_t out_layer_stride, __nv_bfloat16 *k, __nv_bfloat16 *v,
                              cudaStream_t st) {
  const PageList<N> list = list_of<N>(pages, n_pages);
  const dim3 grid(n_pages, layer_count);
  if (pv.head_dim == 128) kv8_read_kernel<128, N><<<grid, A_THREADS, 0, st>>>(pv, list, n_tok, first_offset, layer_begin, out_layer_stride, k, v);
  else kv8_read_kernel<64, N><<<grid, A_THREADS, 0, st>>>(pv, list, n_tok, first_offset, layer_begin, out_layer_stride, k, v);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_append(const PoolView &pv, const int32_t *slots, const int32_t *pos, int32_t n_tok, int32_t layer_begin,
                              int32_t layer_count, int64_t in_layer_stride, const void *k_new, const void *v_new, double theta,
                              cudaStream_t st) {
  if (n_tok == 0 || layer_count == 0) return cudaSuccess;
  const int per = layers_per_cta(n_tok, layer_count);
  const dim3 grid(n_tok, (layer_count + per - 1) / per);
  const Freqs &fr = freqs_of(theta > 0 ? theta : 2.0, pv.head_dim);
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(k_new), *v = static_cast<const __nv_bfloat16 *>(v_new);
#define PASTA_A8(DD, RR) \
  kv8_append_kernel<DD, RR><<<grid, A_THREADS, 0, st>>>(pv, slots, pos, n_tok, layer_begin, layer_count, per, in_layer_stride, k, v, fr)
  if (pv.head_dim == 128) { if (theta > 0) PASTA_A8(128, true); else PASTA_A8(128, false); }
  else { if (theta > 0) PASTA_A8(64, true); else PASTA_A8(64, false); }
#undef PASTA_A8
  return cudaGetLastError();
}

cudaError_t launch_kv8_append_run(const PoolView &pv, const int32_t *pages, int32_t first_offset, int32_t pos0, int32_t n_tok,
                                  int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const void *k_new,
                                  const void *v_new, double theta, cudaStream_t st, int64_t *launches) {
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(k_new), *v = static_cast<const __nv_bfloat16 *>(v_new);
  const int64_t tok = static_cast<int64_t>(pv.n_kv_heads) * pv.head_dim;
  for (int32_t done = 0; done < n_tok;) {
    const int32_t left = n_tok - done, all = (first_offset + left + PASTA_PAGE - 1) / PASTA_PAGE;
    const int32_t n = std::min(all, kPagesLarge), cnt = std::min(left, n * PASTA_PAGE - first_offset);
    const cudaError_t e = n <= kPagesSmall
        ? launch_append_pages<kPagesSmall>(pv, pages, n, pos0 + done, cnt, first_offset, layer_begin, layer_count, in_layer_stride, k + done * tok, v + done * tok, theta, st)
        : launch_append_pages<kPagesLarge>(pv, pages, n, pos0 + done, cnt, first_offset, layer_begin, layer_count, in_layer_stride, k + done * tok, v + done * tok, theta, st);
    if (e != cudaSuccess) return e;
    *launches += 1;
    pages += n;
    done += cnt;
    first_offset = 0;
  }
  return cudaSuccess;
}

cudaError_t launch_kv8_read_run(const PoolView &pv, const int32_t *pages, int32_t first_offset, int32_t n_tok, int32_t layer_begin,
                                int32_t layer_count, int64_t out_layer_stride, void *k_out, void *v_out, cudaStream_t st,
                                int64_t *launches) {
  __nv_bfloat16 *k = static_cast<__nv_bfloat16 *>(k_out), *v = static_cast<__nv_bfloat16 *>(v_out);
  const int64_t tok = static_cast<int64_t>(pv.n_kv_heads) * pv.head_dim;
  for (int32_t done = 0; done < n_tok;) {
    const int32_t left = n_tok - done, all = (first_offset + left + PASTA_PAGE - 1) / PASTA_PAGE;
    const int32_t n = std::min(all, kPagesLarge), cnt = std::min(left, n * PASTA_PAGE - first_offset);
    const cudaError_t e = n <= kPagesSmall
        ? launch_read_pages<kPagesSmall>(pv, pages, n, cnt, first_offset, layer_begin, layer_count, out_layer_stride, k + done * tok, v + done * tok, st)
        : launch_read_pages<kPagesLarge>(pv, pages, n, cnt, first_offset, layer_begin, layer_count, out_layer_stride, k + done * tok, v + done * tok, st);
    if (e != cudaSuccess) return e;
    *launches += 1;
    pages += n;
    done += cnt;
    first_offset = 0;
  }
  return cudaSuccess;
}

}  // namespace pasta
