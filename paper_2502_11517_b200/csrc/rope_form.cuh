// Rotary position embedding: the table of a form (pair layout, rotated part, frequencies), the sines and cosines of a CTA's
// tokens, and the rotation of 16 elements of a row.
//
// A row of head_dim elements is head_dim / 16 slots of 16 elements (two chunks of 8): the elements a[0..7] and b[0..7] of slot
// p turn by the angles of pairs 8 p .. 8 p + 7.  "half" pairs element i with i + R/2, so a slot is chunks p and p + R/16;
// "interleaved" pairs 2 i with 2 i + 1, so a slot is chunks 2 p and 2 p + 1, its elements taken alternately.  Slots behind the
// rotated part (p >= R/16) are chunks 2 p and 2 p + 1 under either layout and turn by nothing: their cosine is exactly 1.
//
// Angles, sines, cosines and products are 64-bit, the result is rounded to fp32 once (and by the caller to what it stores).
// Sines and cosines are kept times 2^896, and a bf16 number becomes the 64-bit number whose exponent field is its own: that
// is the number times 2^-896, subnormal or not, for two integer instructions in place of a conversion (measured: 17 cycles
// per warp for a conversion there and back, 2 for a multiplication).
#pragma once
#include "device_common.cuh"

namespace pasta {

struct RopeForm {
  double f[64], c1[64], s1[64];      // frequency of pair i; the rotation by one position is (c1[i], s1[i])
  double size;                       // what rotated elements are multiplied by
  int32_t slots;                     // R / 16
  int32_t interleaved;
};

// the whole head, first half paired with second, nothing multiplied
inline bool rope_form_is_plain(const RopeForm &f, int head_dim) { return f.slots * 16 == head_dim && !f.interleaved && f.size == 1.0; }

constexpr double kTurnScale = 0x1p896;
__device__ __forceinline__ double scaled_down(uint32_t bits) {       // bits: fp32 bits of a bf16 number
  return __hiloint2double((static_cast<int>(bits) >> 3) & 0x8fffffff, 0);
}

__device__ __forceinline__ int rope_chunk_a(const RopeForm &f, int p) { return p < f.slots && !f.interleaved ? p : 2 * p; }
__device__ __forceinline__ int rope_chunk_b(const RopeForm &f, int p) { return p < f.slots && !f.interleaved ? p + f.slots : 2 * p + 1; }

// (cos, sin) of pair i = 8 p + e of a token at turn[e * (D / 16) + p]
template <int D>
__device__ __forceinline__ int turn_at(int i) { return (i & 7) * (D / 16) + (i >> 3); }
__device__ __forceinline__ double2 turn_of(const RopeForm &f, int i, int pos) {
  if (i >= 8 * f.slots) return make_double2(kTurnScale, 0.0);
  double sn, cs;
  sincos(static_cast<double>(pos) * f.f[i], &sn, &cs);
  return make_double2(cs * f.size * kTurnScale, sn * f.size * kTurnScale);
}

// The same for `cnt` (<= 16) consecutive positions from pos0 on, into turn[r * D/2 + ...], by a CTA of kThreads threads: a
// thread works out the sine and cosine of one angle at every fourth token and turns it on by one position at a time for the
// three behind it: three products, each good to a few times 2^-53.
template <int D, int kThreads>
__device__ __forceinline__ void turns_of_run(const RopeForm &f, int pos0, int cnt, double2 *turn) {
  constexpr int H = D / 2;
  for (int x = threadIdx.x; x < PASTA_PAGE / 4 * H; x += kThreads) {
    const int r = x / H * 4, i = x % H;
    if (r >= cnt) break;
    double2 t = turn_of(f, i, pos0 + r);
    const double c1 = i < 8 * f.slots ? f.c1[i] : 1.0, s1 = i < 8 * f.slots ? f.s1[i] : 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (r + j < cnt) turn[(r + j) * H + turn_at<D>(i)] = t;
      t = make_double2(t.x * c1 - t.y * s1, t.y * c1 + t.x * s1);
    }
  }
}

// Slot p of a row: lo and hi are its chunks a and b as loaded, all numbers finite; y[e] and y[8 + e] are the rotated elements
// a[e] and b[e].  alternate: the elements are taken alternately (a rotated slot of the interleaved layout).
template <int D>
__device__ __forceinline__ void rope_slot(const uint4 &lo4, const uint4 &hi4, bool alternate, const double2 *turn, int p, float *y) {
  const uint32_t w[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // the pair's elements: the two halves of one word, or the same half of words e / 2 of either chunk
    const uint32_t wa = alternate ? w[e] << 16 : (e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16;
    const uint32_t wb = alternate ? w[e] & 0xffff0000u : (e & 1) ? w[4 + (e >> 1)] & 0xffff0000u : w[4 + (e >> 1)] << 16;
    const double a = scaled_down(wa), b = scaled_down(wb);
    const double2 t = turn[e * (D / 16) + p];
    y[e] = static_cast<float>(a * t.x - b * t.y);
    y[8 + e] = static_cast<float>(b * t.x + a * t.y);
  }
}

// any number of a chunk that is not finite
__device__ __forceinline__ bool chunk_not_finite(const uint4 &x) {
  const uint32_t m2 = __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
  return (m2 & 0xffffu) >= 0x7f80u || m2 >= 0x7f800000u;
}
// Numbers that are not finite become zeros, and with them what they are paired with (turns: the slot is a rotated one).
__device__ __forceinline__ void rope_clean(uint4 &lo4, uint4 &hi4, bool alternate, bool turns) {
  uint32_t *lo = reinterpret_cast<uint32_t *>(&lo4), *hi = reinterpret_cast<uint32_t *>(&hi4);
  auto keep = [](uint32_t x) { return ((x & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u); };
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t kl = keep(lo[w]), kh = keep(hi[w]);
    if (alternate) {
      kl = kl == 0xffffffffu ? kl : 0u;
      kh = kh == 0xffffffffu ? kh : 0u;
    } else if (turns) {
      kl = kh = kl & kh;
    }
    lo[w] &= kl;
    hi[w] &= kh;
  }
}
// The chunks a slot's rotated elements go back to.
__device__ __forceinline__ void rope_unslot(const float *y, bool alternate, float *lo, float *hi) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo[j] = alternate ? y[(j & 1) * 8 + (j >> 1)] : y[j];
    hi[j] = alternate ? y[(j & 1) * 8 + 4 + (j >> 1)] : y[8 + j];
  }
}

}  // namespace pasta
