// Device-side helpers shared by the kernels: pool layout, mbarrier / bulk-copy wrappers, bounded waits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/pasta.h"
#include "pasta_plan.h"

namespace pasta {

// ---------------------------------------------------------------------------------------------
// Layout of one (page, kv head) block of the pool: K and V of 16 tokens, D*64 bytes.
//
//   block = [token group j: 2][K, V: 2][64-element half of the head dim: D/64][8 rows x 128 bytes]
//
// Each 1024-byte atom holds 8 tokens x 64 bf16; inside it the 16-byte chunk c of row r sits at
// chunk position c ^ r (the 128-byte swizzle the tensor core reads), so that one bulk copy of a
// block lands in shared memory ready to be used as an MMA operand: K as a K-major operand with
// rows = tokens, V as an MN-major operand with the head dim along N.  The same swizzle makes
// "one token per lane" reads of shared memory bank-conflict free in the warp-shuffle kernel.
// ---------------------------------------------------------------------------------------------
__host__ __device__ constexpr int kv_block_bytes(int head_dim) { return head_dim * 64; }

// byte offset, inside a block, of the 16-byte chunk `c` (8 elements) of token row `r` (0..15);
// kv = 0 for K, 1 for V; NH = head_dim / 64
__device__ __forceinline__ int kv_chunk_offset(int NH, int kv, int r, int c) {
  const int j = r >> 3, r8 = r & 7, half = c >> 3, c8 = c & 7;
  return (((j * 2 + kv) * NH + half) << 10) + (r8 << 7) + ((c8 ^ r8) << 4);
}

// ---------------------------------------------------------------------------------------------
// Layout of one (page, kv head) block of an 8-bit pool (PASTA_FLAG_KV_FP8): e4m3 codes of K and V of 16 tokens,
// D*32 bytes, one byte per element:
//
//   block = [token group j: 2][K, V: 2][8 rows x D bytes]
//
// A row holds one token's codes in 16-byte chunks; chunk c of row r (0..7) sits at chunk position c ^ r for D = 128 and at
// c ^ (r >> 1) for D = 64 (the 128- and 64-byte swizzles), which keeps both ways the attention kernels read a block
// free of bank conflicts: a lane per token along a row (K), and 16 tokens of one chunk at a time (V, transposed).
// Behind a layer's blocks lie its scales: two signed bytes per (page, kv head), the exponents ek and ev of the page's
// K and V; an element is code * 2^e.  Codes are never NaN (the append stores no such code), so bytes of a page beyond a
// stream's end, whatever they are, vanish against zero weights.
// ---------------------------------------------------------------------------------------------
__host__ __device__ constexpr int kv8_block_bytes(int head_dim) { return head_dim * 32; }
constexpr int kKv8ExpMin = -64, kKv8ExpMax = 63;     // range of a page's scale exponent

// byte offset, inside an 8-bit block, of the 16-byte chunk `c` (16 elements) of token row `r` (0..15)
template <int D>
__device__ __forceinline__ int kv8_chunk_offset(int kv, int r, int c) {
  const int j = r >> 3, r8 = r & 7;
  return (j * 2 + kv) * (8 * D) + r8 * D + ((c ^ (D == 128 ? r8 : (r8 >> 1))) << 4);
}

struct PoolView {
  uint8_t *kv_base;
  int64_t layer_stride;      // bytes between layers
  int32_t n_pages, n_q_heads, n_kv_heads, head_dim;
  int32_t *status;           // device status word
  const int32_t *plan;       // device copy of the step plan
  float2 *part_ml;           // partial (m, l) per row; m in log2 units of the scaled score
  float *part_o;             // partial unnormalised outputs [row][D]
  int64_t rows_per_layer;    // stride of the partial arrays between layers of one launch
  long long wait_limit;      // SM cycles a role waits for another role before it gives up (kWaitLimitCycles by default)
  float softcap_log2;        // 0, or C = cap * log2(e): a score s (in log2 units) becomes C tanh(s / C)
  int32_t kv8;               // 1: the pool holds 8-bit codes and scales (kv8_block_bytes, kv8_chunk_offset)
  int64_t scale_off;         // bytes from a layer's start to its scales (8-bit pools)
  int32_t debug_hold;        // test hook, 0 in normal use: bit r set = role r of the tensor-core kernel never starts
};

__device__ __forceinline__ void report(int32_t *status, int32_t code) { atomicMax(status, code); }
// The status word is the first of 64 words the library keeps for itself.  Word 8 counts the shared units the CTAs of
// the tensor-core kernel have taken in the current launch (the merge that follows puts it back to zero); words 16-17
// are the sink of the read-only measurement kernels.
#define PASTA_STATUS_TAIL_COUNTER 8

// Overlap of consecutive launches of a step (programmatic dependent launch).  A kernel launched with launch_overlapped()
// may start while the kernel before it in the stream is still running, once every CTA of that kernel has called
// grid_launch_dependents() or has exited; it must call grid_dependency_wait(), in every thread and before its first
// access to anything the earlier kernel reads or writes, which returns when the earlier kernel has completed and its
// writes are visible.  What runs before that call (barrier set-up, TMEM allocation, the launch itself) is hidden behind
// the earlier kernel's last CTAs.  Each kernel waits before it lets its own successor go, so that the completion of a
// kernel implies that of all its predecessors.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_init_fence() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void fence_proxy_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// the same look at a phase without waiting at all (try_wait may suspend the thread for a while)
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Default upper bound of every wait inside a kernel, in SM clock cycles (about 1.5 s at 2 GHz).  Waits of one role
// for another take the pool's limit (PoolView::wait_limit, this value unless a test shortened it); waits for the
// hardware to finish what the CTA itself started (bulk copies, MMAs in flight when a role gives up) always take
// this constant: they end on their own.
constexpr long long kWaitLimitCycles = 3000000000ll;

// Waits for the phase with the given parity to complete, for at most `limit` cycles.
// Returns false when the wait was given up (the caller then reports PASTA_ERR_TIMEOUT and leaves).
__device__ __forceinline__ bool mbar_wait_bounded(uint32_t bar, uint32_t parity, long long limit = kWaitLimitCycles) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 256; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (clock64() - t0 > limit) return false;
  }
}

// 1-D bulk copy global -> shared, completion counted in bytes on an mbarrier.
// Both addresses 16-byte aligned, size a multiple of 16.
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
      ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// tanh(x) / x for u = x^2 <= 1: the interpolation at seven Chebyshev nodes of [0, 1], off by less than 2^-24 (2^-23 as evaluated
// in fp32), highest power first.
#define PASTA_TANH_POLY(STEP) \
  STEP(-6.1943247e-3f) STEP(2.0279707e-2f) STEP(-5.3451646e-2f) STEP(0.13325076f) STEP(-0.33332828f) STEP(0.99999994f)
constexpr float kTanhPolyTop = 1.0380251e-3f;
// Capped score C tanh(x), x = s / C, as 1 - 2 / (2^(2 x log2 e) + 1): ex2 and rcp are good to a few units of the last place, so
// the result is off by less than 2^-21 C whatever x is.  Saturates to +-C.
__device__ __forceinline__ float softcap_any(float x, float C) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fast_exp2(x * (2.f * 1.4426950408889634f)) + 1.f));
  return fmaf(-2.f * C, r, C);
}
// The same with the polynomial up to |x| = 1: good to 2^-22 of the result there, so that a cap far above the scores leaves them
// as they are.
__device__ __forceinline__ float softcap(float x, float C) {
  if (fabsf(x) > 1.f) return softcap_any(x, C);
  const float u = x * x;
  float t = kTanhPolyTop;
#define PASTA_STEP(c) t = fmaf(t, u, c);
  PASTA_TANH_POLY(PASTA_STEP)
#undef PASTA_STEP
  return t * x * C;
}

// two e4m3 codes (low and high byte of a 16-bit half of `x`) as two fp16: exact
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t x) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(x));
  return r;
}
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t x, uint32_t &lo, uint32_t &hi) {
  lo = e4m3x2_to_f16x2(static_cast<uint16_t>(x));
  hi = e4m3x2_to_f16x2(static_cast<uint16_t>(x >> 16));
}
// nearest e4m3 codes of four numbers (ties to even, magnitudes above 448 held there), a in the lowest byte
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
// 2^e as fp32 for -126 <= e <= 127
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }
// What takes the place of a row's (reference, sum) on 8-bit pools when its query holds a number that is not finite: the merge
// gives it all the weight, its accumulator is NaN, and so is the output (lse is infinite).
__device__ __forceinline__ float2 not_a_row() { return make_float2(3.4e38f, INFINITY); }
// What a score over codes is multiplied by: the row's factor and K's scale, kept off infinity so that a score of 0 stays 0
// (8-bit pools; only reached where the scores of anything but 0 leave fp32's range).
__device__ __forceinline__ float code_factor(float row, int ek) { return fminf(row * pow2f(ek), 1e38f); }
// The same over the cap, which may be far below 1.
__device__ __forceinline__ float capped_factor(float c, float cap_inv) { return fminf(c * cap_inv, 1e38f); }

}  // namespace pasta
