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

struct Freqs { double f[64]; };          // theta^(-2i/D)

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

// One CTA per page group (the new tokens that fall into one page) and slice of the layers; a warp takes one (kv head, K or
// V) at a time, holds the group's elements in registers, finds their largest magnitude, and writes the codes: every
// element is read once.  The rotation's sines and cosines (64 bits) are worked out once per CTA for all heads and layers.
template <int D, bool kRope>
__global__ void __launch_bounds__(A_THREADS)
kv8_append_kernel(PoolView pv, const int32_t *__restrict__ slots, const int32_t *__restrict__ pos, int32_t pos0, int32_t n_tok,
                  int32_t consecutive, int32_t first_offset, int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta,
                  int64_t in_layer_stride, const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new,
                  Freqs freqs) {
  constexpr int H = D / 2;
  __shared__ double2 turn[kRope ? PASTA_PAGE * H : 1];       // (cos, sin) of token r, angle i = 8 c + e at r * H + e * (H / 8) + c
  grid_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int first, cnt;
  if (consecutive) {
    first = max(0, static_cast<int>(blockIdx.x) * PASTA_PAGE - first_offset);
    cnt = min(n_tok, (static_cast<int>(blockIdx.x) + 1) * PASTA_PAGE - first_offset) - first;
  } else {
    // the CTA of a group's first token takes the group: a token continues one if its slot is the next of the same page
    first = blockIdx.x;
    const int page = slots[2 * first], off = slots[2 * first + 1];
    if (first > 0 && slots[2 * first - 2] == page && slots[2 * first - 1] == off - 1) return;
    const int a = first + lane;
    const bool mine = lane < PASTA_PAGE && a < n_tok && slots[2 * a] == page && slots[2 * a + 1] == off + lane;
    cnt = __ffs(~__ballot_sync(0xffffffffu, mine)) - 1;
  }
  const int page = slots[2 * first], off0 = slots[2 * first + 1];
  if (page < 0 || page >= pv.n_pages || off0 < 0 || off0 + cnt > PASTA_PAGE || cnt < 1) {
    if (tid == 0) report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  if (kRope) {
    for (int x = tid; x < cnt * H; x += A_THREADS) {
      const int r = x / H, i = x % H;
      double sn, cs;
      sincos(static_cast<double>(pos ? pos[first + r] : pos0 + first + r) * freqs.f[i], &sn, &cs);
      turn[r * H + (i & 7) * (H / 8) + (i >> 3)] = make_double2(cs, sn);
    }
    __syncthreads();
  }
  const int Hkv = pv.n_kv_heads;
  const int ll_end = min(layer_count, (static_cast<int>(blockIdx.y) + 1) * layers_per_cta);
  for (int ll = blockIdx.y * layers_per_cta; ll < ll_end; ++ll) {
    uint8_t *layer = pv.kv_base + (layer_begin + ll) * pv.layer_stride;
    for (int item = warp; item < 2 * Hkv; item += A_WARPS) {
      const int g = item >> 1, kv = item & 1;
      const __nv_bfloat16 *src = (kv ? v_new : k_new) + ll * in_layer_stride + (static_cast<int64_t>(first) * Hkv + g) * D;
      const int64_t at = static_cast<int64_t>(page) * Hkv + g;
      uint8_t *block = layer + at * kv8_block_bytes(D);
      int8_t *scale = reinterpret_cast<int8_t *>(layer + pv.scale_off) + at * 2 + kv;
      bool bad = false;
      if (kRope && kv == 0) {
        // a lane holds the 8 elements of chunk c of the low half and the 8 they pair with in the high half
        constexpr int LPT = D / 16, TPI = 32 / LPT, NI = PASTA_PAGE / TPI;
        const int c = lane % LPT;
        float y[NI][16];
        uint32_t amax = 0;
#pragma unroll
        for (int it = 0; it < NI; ++it) {
          const int r = it * TPI + lane / LPT;
          if (r < cnt) {
            const uint4 *row = reinterpret_cast<const uint4 *>(src + static_cast<int64_t>(r) * Hkv * D);
            const uint4 lo4 = __ldg(row + c), hi4 = __ldg(row + c + LPT);
            const uint32_t lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const double2 t = turn[r * H + e * (H / 8) + c];
              const double a = (e & 1) ? bf16_hi(lo[e >> 1]) : bf16_lo(lo[e >> 1]);
              const double b = (e & 1) ? bf16_hi(hi[e >> 1]) : bf16_lo(hi[e >> 1]);
              y[it][e] = static_cast<float>(a * t.x - b * t.y);
              y[it][8 + e] = static_cast<float>(b * t.x + a * t.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[it][e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if ((__float_as_uint(y[it][e]) & 0x7fffffffu) >= 0x7f800000u) { y[it][e] = 0.f; bad = true; }
            amax = max(amax, __float_as_uint(y[it][e]) & 0x7fffffffu);
          }
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
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

// One thread per 8 elements of one (token, kv head, K or V): 8 bytes in, 16 bytes out.  blockIdx.y = layer.
template <int D>
__global__ void __launch_bounds__(256)
kv8_read_kernel(PoolView pv, const int32_t *__restrict__ slots, int32_t n_tok, int32_t layer_begin, int64_t out_layer_stride,
                __nv_bfloat16 *__restrict__ k_out, __nv_bfloat16 *__restrict__ v_out) {
  constexpr int CH = D / 8;
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int c = static_cast<int>(idx % CH);
  const int64_t row = idx / CH;                     // (kv, token, head)
  const int64_t per = static_cast<int64_t>(n_tok) * pv.n_kv_heads;
  if (row >= 2 * per) return;
  const int kv = row >= per;
  const int64_t th = row - kv * per;
  const int a = static_cast<int>(th / pv.n_kv_heads), g = static_cast<int>(th % pv.n_kv_heads);
  const int page = slots[2 * a], off = slots[2 * a + 1];
  if (page < 0 || page >= pv.n_pages || off < 0 || off >= PASTA_PAGE) {
    report(pv.status, PASTA_ERR_DEVICE_CHECK);
    return;
  }
  const uint8_t *layer = pv.kv_base + (layer_begin + static_cast<int64_t>(blockIdx.y)) * pv.layer_stride;
  const int64_t at = static_cast<int64_t>(page) * pv.n_kv_heads + g;
  const float f = pow2f(*(reinterpret_cast<const int8_t *>(layer + pv.scale_off) + at * 2 + kv));
  const uint2 q = *reinterpret_cast<const uint2 *>(layer + at * kv8_block_bytes(D) + kv8_chunk_offset<D>(kv, off, c >> 1) + (c & 1) * 8);
  uint32_t h[4], o[4];
  e4m3x4_to_f16x4(q.x, h[0], h[1]);
  e4m3x4_to_f16x4(q.y, h[2], h[3]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h[w]));
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * f, v.y * f);      // exact: four significant bits
    o[w] = *reinterpret_cast<const uint32_t *>(&b);
  }
  __nv_bfloat16 *dst = (kv ? v_out : k_out) + blockIdx.y * out_layer_stride + th * D + c * 8;
  *reinterpret_cast<uint4 *>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
}

}  // namespace

cudaError_t launch_kv8_append(const PoolView &pv, const int32_t *slots, const int32_t *pos, int32_t pos0, int32_t n_tok,
                              bool consecutive, int32_t first_offset, int32_t layer_begin, int32_t layer_count,
                              int64_t in_layer_stride, const void *k_new, const void *v_new, double theta, cudaStream_t st) {
  if (n_tok == 0 || layer_count == 0) return cudaSuccess;
  const int groups = consecutive ? (first_offset + n_tok + PASTA_PAGE - 1) / PASTA_PAGE : n_tok;
  // all layers of a group in one CTA share its sines and cosines; split them only as far as the GPU has to be filled
  const int want = 148 * 4;
  const int slices = std::min(layer_count, std::max(1, (want + groups - 1) / groups));
  const int per = (layer_count + slices - 1) / slices;
  const dim3 grid(groups, (layer_count + per - 1) / per);
  Freqs fr{};
  if (theta > 0)
    for (int i = 0; i < pv.head_dim / 2; ++i) fr.f[i] = std::exp2(-2.0 * i / pv.head_dim * std::log2(theta));
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(k_new), *v = static_cast<const __nv_bfloat16 *>(v_new);
#define PASTA_A8(DD, RR)                                                                                                     \
  kv8_append_kernel<DD, RR><<<grid, A_THREADS, 0, st>>>(pv, slots, pos, pos0, n_tok, consecutive ? 1 : 0, first_offset,       \
                                                        layer_begin, layer_count, per, in_layer_stride, k, v, fr)
  if (pv.head_dim == 128) { if (theta > 0) PASTA_A8(128, true); else PASTA_A8(128, false); }
  else { if (theta > 0) PASTA_A8(64, true); else PASTA_A8(64, false); }
#undef PASTA_A8
  return cudaGetLastError();
}

cudaError_t launch_kv_read_layers(const PoolView &pv, const int32_t *slots, int32_t n_tok, int32_t layer_begin,
                                  int32_t layer_count, int64_t out_layer_stride, void *k_out, void *v_out, cudaStream_t st) {
  if (n_tok == 0 || layer_count == 0) return cudaSuccess;
  __nv_bfloat16 *k = static_cast<__nv_bfloat16 *>(k_out), *v = static_cast<__nv_bfloat16 *>(v_out);
  if (!pv.kv8) {
    for (int32_t l = 0; l < layer_count; ++l) {
      const cudaError_t e = launch_kv_read(pv, slots, n_tok, layer_begin + l, k + l * out_layer_stride, v + l * out_layer_stride, st);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  const int64_t threads = 2 * static_cast<int64_t>(n_tok) * pv.n_kv_heads * (pv.head_dim / 8);
  const dim3 grid(static_cast<unsigned>((threads + 255) / 256), layer_count);
  if (pv.head_dim == 128) kv8_read_kernel<128><<<grid, 256, 0, st>>>(pv, slots, n_tok, layer_begin, out_layer_stride, k, v);
  else kv8_read_kernel<64><<<grid, 256, 0, st>>>(pv, slots, n_tok, layer_begin, out_layer_stride, k, v);
  return cudaGetLastError();
}

}  // namespace pasta
