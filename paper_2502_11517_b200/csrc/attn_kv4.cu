// K2 of a 4-bit pool, head_dim 64 and 128: tensor-core pass over 4-bit codes (the plan, units and rows are those of
// attn_tensor.cu; the layout of a block is described in device_common.cuh).
//
//   S^T[128 tokens x N] = K[128 x D] . Q^T          tcgen05.mma kind::f16, A = K from TMEM, B = the stacked queries
//   P^T                 = 2^(S^T scale*log2e - ref)  a thread per token; ref per row, capped and masked where asked for
//   O^T[D x N]         += V^T[D x 128] . P^T         A = V^T from TMEM, B = the weights (bf16) in shared memory
//   l                  += P^T, summed over tokens     out = O / l
//
// N is the number of stacked rows (threads x group) rounded up to 16.  Tokens lie along M and rows along N, the other way
// round than in attn_tensor.cu, because that is what 4-bit codes ask for: (1) codes have to become bf16 numbers (kv4_value:
// exact) before they can be multiplied, and as the A operand they go straight from the registers of the thread that converts them
// into tensor memory, a thread per token for K and a thread per channel for V, without a round trip through shared memory;
// (2) a step has few rows (4 per thread of a response), and every instruction of the softmax, every exponential and every cycle
// of the tensor pipe is spent on N columns instead of 128.
//
// head_dim 64 has 64 channels for the 128 rows of O^T's MMA, so V^T's upper 64 rows are the channels of the tile's second 64
// tokens, and the weights of those tokens are N further columns: [V_0; V_1] [P_0 | P_1], K = 64 (the columns of P_0 and P_1 eight
// at a time in turn).  The two diagonal blocks are what is wanted and are added up at a unit's end; the other two cost nothing
// that matters at these N.
//
// What bounds it: instructions and their latency.  A tile of 128 tokens and 68 rows takes 7100 warp instructions (a quarter to each
// scheduler: some 1800, of which K's codes, V's codes and the softmax are 1000), against the 785 cycles that its 18 KB take at the
// measured copy bandwidth.  A warp alone issues one every seven cycles, and a tile is a chain (codes, MMA, codes and softmax, MMA), so
// CTAs share an SM and fill one another's gaps: four of 128 threads and 128 TMEM columns for up to 32 rows, two of 256 threads and
// 256 columns for up to 80 (64 at head_dim 64); requests with more rows are split by the planner.  Schedulers issue in 55 % of the cycles; a tile takes 2500
// (68 rows) to 1700 (20 rows) cycles of an SM.  Measured: 64 requests of 4 to 36 rows 155 us (39 us for the bytes alone), 8 prefixes of
// 32768 tokens and 68 rows 239 us (52), 64 capped short responses 159 us (24), 32 requests of 2 to 10 rows at head_dim 64 46 us (7).
// Built and measured slower: roles on warps of their own and one CTA to an SM, in three forms (290 to 390 us for the first, 310 to 410
// for the second: hand-overs and four programs' instruction fetches); twice the threads per CTA at 64 registers (302 and 418); bulk
// copies in place of 16-byte ones (192 and 277 for 191 and 274 then); one body for the chunks of the softmax instead of one for
// every number of them (154 and 243 for 152 and 236).
//
// A CTA walks units as those of attn_tensor.cu do, but where runs are short they are handed out at run time, whole, the longest first.  TMEM holds one
// operand (K, then V in its place), the scores and O^T.  Every warp does everything in turn.
// References: a weight is 2^(score - ref), and any ref that keeps weights, and their products with values, inside the range of fp32 and bf16
// (which share their exponents) gives the same relative precision.  So a row's ref starts at 0 and nobody looks for maxima.  When a score exceeds its row's ref by
// more than R_SLACK (the CTA votes on that with the barrier that publishes the weights), the rows' maxima over the tile are worked out, and
// O and l brought to them.  A row that saw tokens but whose sum came out below 2^-60 has scores far below 0: its unit is done again,
// with first references from the maxima of the first tokens each row sees.
// A reference is a score rounded to fp32, and what a score exceeds it by comes out of one multiply-add, unrounded.  The two differ by half a
// step of the score: nothing near 0, but whole powers of two from 2^24 on, and from 2^31 weights that are infinite, or all zero.  So the unit
// of a row with a reference beyond R_FAR is done again without tensor cores (plain_rows), where a row's largest score is exactly its
// reference.  The same where values next to the range's upper end, under many weights, add up to more than fp32 or the merge holds; rows whose
// weights are small and whose values are so too that products may have been lost (all of O below 2^-110) are done again carefully.  O is looked at for
// that only where the weights' sums allow either.
// (Rounded products beside the others on the tensor path cost every step 3 to 7 % for want of registers.)
// The threads that share a token (or channel) share its groups of channels, its pages and its chunks of eight rows.
// Every wait is bounded; on expiry the CTA reports PASTA_ERR_TIMEOUT, drains and leaves.
#include <algorithm>
#include <type_traits>

#include "tensor_common.cuh"

namespace pasta {

namespace {

constexpr float R_SLACK = 10.f;                  // weights are at most 2^10 (bf16 and fp32 keep their precision at any size)
constexpr float R_FAR = 16777216.f;              // 2^24: beyond it a score and its rounding differ by whole powers of two
constexpr float R_UNSET = 3e38f;                 // minus the reference of a row that has seen nothing (careful units)
// Sums of weighted values: at most so much in partial rows (the merge adds up some 2^9 of them), and at least so much in a row's largest, or
// products may have been lost.  Values are below 2^114, so what the weights' sum is tells where a row can be outside.
constexpr float O_PART = 0x1p118f, O_TINY = 0x1p-110f;
constexpr float L_PART = 0x1p4f, L_FINAL = 0x1p14f, L_TINY = 0x1p-16f;
constexpr float R_FAINT = 8.7e-19f;              // 2^-60: sums below it may have lost weights to fp32's range

// Sizes of one build: head_dim D, at most NMAX stacked rows.
template <int D, int NMAX>
struct U {
  static constexpr int H = NMAX <= 32 ? 1 : 2, THREADS = 128 * H;      // threads that share a token
  static constexpr int CHUNKS = NMAX / 8 / H;                     // groups of 8 rows per thread, at most: chunk H i + part for its part
  static_assert(NMAX % (8 * H) == 0 && CHUNKS <= 5, "numbers of chunks");
  static constexpr int OW = D == 128 ? 1 : 2;                     // blocks of N columns of an accumulator
  static constexpr int KSTEPS = D / 16, VSTEPS = D == 128 ? 8 : 4;
  static constexpr uint32_t COL_A = 0, COL_S = D / 2, COL_O = COL_S + NMAX;      // (V's operand is D / 2 columns wide, too)
  static constexpr uint32_t COLS_USED = COL_O + OW * NMAX, COLS = COLS_USED <= 128 ? 128 : 256;
  static_assert(COLS_USED <= 256, "tensor memory budget");
  static constexpr int RESIDENT = 512 / COLS;                     // CTAs on an SM
  static constexpr int BLOCK = kv4_block_bytes(D), STAGE_BYTES = PASTA_TILE_PAGES * BLOCK;
  static constexpr int STAGES = D == 128 && NMAX <= 32 ? 2 : 3;
  // a row of weights: 128 bytes per 64 columns, or 64 bytes where they are at most 32 (so that four CTAs fit)
  static constexpr bool NARROW = OW * NMAX <= 32;
  static constexpr int ATOMS = (OW * NMAX + 63) / 64, P_GROUP = NARROW ? 512 : ATOMS * 1024;      // bytes of 8 rows
  static constexpr int P_BYTES = (D == 128 ? 16 : 8) * P_GROUP;
  static constexpr int Q_BYTES = NMAX * D * 2;
  // (head_dim 64: the halves of accumulators are added up where the weights were)
  static_assert(D == 128 || NMAX * 64 * 4 <= P_BYTES, "room for 64 channels of every row");
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_P = OFF_Q + Q_BYTES;
  static constexpr int OFF_STAGE = OFF_P + P_BYTES;
  static constexpr int OFF_BAR = OFF_STAGE + STAGES * STAGE_BYTES;
  static constexpr int B_QK = 0, B_PV = 1, B_DRAIN = 2, B_COUNT = 3;
  static constexpr int OFF_META = OFF_BAR + 8 * ((B_COUNT + 1) & ~1);    // [STAGES] 8 page metas
  static constexpr int OFF_MISC = OFF_META + STAGES * 32;                // tmem base, abort flag, -, -, the unit's record
  static constexpr int OFF_REF = OFF_MISC + 16 + 64;                     // [NMAX] references (negated)
  static constexpr int OFF_FACT = OFF_REF + NMAX * 4;                    // [NMAX] what a raised reference multiplies O and l by; 1 / l
  static constexpr int OFF_WARP = OFF_FACT + NMAX * 4;                   // [4][NMAX] a warp's maxima, or sums
  static constexpr int OFF_SEEN = OFF_WARP + 4 * NMAX * 4;               // [4][8] threads that see something in the tile, by its quarters (16 a word),
                                                                         // then [4][8] in the whole unit, and [8] that wait for that
  static constexpr int SMEM_BYTES = OFF_SEEN + (32 + 32 + 8) * 4 + 1024; // slack to align the base to 1024
  static_assert((SMEM_BYTES + 1024) * RESIDENT <= 233472, "shared memory budget");
  static_assert(OFF_P % 1024 == 0 && OFF_STAGE % 16 == 0 && OFF_META % 16 == 0 && OFF_MISC % 16 == 0, "alignment");
};

constexpr uint32_t IDESC4 = (1u << 4) | (1u << 7) | (1u << 10) | IDESC_M128;      // D fp32, A and B bf16, M = 128
constexpr uint32_t IDESC4_PV = IDESC4 | (1u << 16);                                // B (= P^T) MN-major

// descriptor of the weights where their rows are 64 bytes: the 64-byte swizzle
__device__ __forceinline__ uint64_t smem_desc64(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return (smem_desc(addr, lbo_bytes, sbo_bytes) & ~(7ull << 61)) | (4ull << 61);
}
__device__ __forceinline__ void tmem_ld8_issue(uint32_t taddr, uint32_t *r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr) : "memory");
}
#define PASTA_RW8(r) "+r"((r)[0]), "+r"((r)[1]), "+r"((r)[2]), "+r"((r)[3]), "+r"((r)[4]), "+r"((r)[5]), "+r"((r)[6]), "+r"((r)[7])
// the wait for every load in flight, and for further sets the promise that nothing that uses them is scheduled above it
__device__ __forceinline__ void tmem_ld_wait8(uint32_t *r) { asm volatile("tcgen05.wait::ld.sync.aligned;" : PASTA_RW8(r) :: "memory"); }
__device__ __forceinline__ void tmem_ld_order8(uint32_t *r) { asm volatile("" : PASTA_RW8(r) :: "memory"); }
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ uint64_t two_floats(float a, float b) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
// {x0, x1} = {x0, x1} * s + {c0, c1}
__device__ __forceinline__ void fma2s(float &x0, float &x1, uint64_t s, float c0, float c1) {
  asm("{\n\t.reg .b64 x, c;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 c, {%3, %4};\n\tfma.rn.f32x2 x, x, %2, c;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(x0), "+f"(x1) : "l"(s), "f"(c0), "f"(c1));
}
// {l0, l1} += the two bf16 numbers of w
__device__ __forceinline__ void add_bf16x2(float &l0, float &l1, uint32_t w) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.bf16 %0, a, %0;\n\tadd.rn.f32.bf16 %1, b, %1;\n\t}" : "+f"(l0), "+f"(l1) : "r"(w));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// Sums of eight numbers over the warp: lane (a b c . .) ends up with the sum of number 4 a + 2 b + c.
__device__ __forceinline__ float warp_sum8(const float *v, int lane) {
  float w[4], u[2], t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float send = (lane & 16) ? v[i] : v[4 + i], keep = (lane & 16) ? v[4 + i] : v[i];
    w[i] = keep + __shfl_xor_sync(0xffffffffu, send, 16);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float send = (lane & 8) ? w[i] : w[2 + i], keep = (lane & 8) ? w[2 + i] : w[i];
    u[i] = keep + __shfl_xor_sync(0xffffffffu, send, 8);
  }
  {
    const float send = (lane & 4) ? u[0] : u[1], keep = (lane & 4) ? u[1] : u[0];
    t = keep + __shfl_xor_sync(0xffffffffu, send, 4);
  }
  t += __shfl_xor_sync(0xffffffffu, t, 2);
  return t + __shfl_xor_sync(0xffffffffu, t, 1);
}

__device__ __forceinline__ bool is_far(float ref) { return fabsf(ref) >= R_FAR && fabsf(ref) < INFINITY && ref != R_UNSET; }

// one lane of a whole warp, the same one every time
__device__ __forceinline__ bool elect_lane() {
  uint32_t y;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(y));
  return y != 0;
}

// 16 bytes from global to shared memory, not kept in L1 and the first to leave L2
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Waits for a phase, or for some thread of the CTA to have given up; sets the flag when the time is up.  Whole warps.
__device__ __forceinline__ void cta_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, long long limit) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
  long long t0 = 0;
#pragma unroll 1
  for (int i = 0; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++i) {
    if (i & 31) continue;
    if (t0 == 0) t0 = clock64();
    if (clock64() - t0 > limit) *abort_flag = 1;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return;
  }
}

// A unit's rows without tensor cores, a warp to a row: a lane has half of a token's channels for the scores, and D / 32 channels
// of V.  o is kept as the mean of the values so far, so nothing leaves the range of what is held.
template <int D, int kWarps, bool kCap>
__device__ __forceinline__ void plain_rows(const PoolView &pv, const TensorArgs &a, const __nv_bfloat16 *q, const UnitInfo &x, int layer) {
  constexpr int E = D / 32, BLOCK = kv4_block_bytes(D);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = pv.n_q_heads / pv.n_kv_heads, g_shift = 31 - __clz(G);
  const int32_t *plan = pv.plan;
  const uint8_t *head = pv.kv_base + (a.layer_begin + layer) * pv.layer_stride + static_cast<int64_t>(x.g) * BLOCK;
  const int last = min(x.tile_end * PASTA_TILE_PAGES, x.n_pages), r = lane & 15;
#pragma unroll 1
  for (int row = warp; row < x.n_threads << g_shift; row += kWarps) {
    const int thread = row >> g_shift, qn = plan[a.off_tq + x.tq_off + thread];
    const int64_t at = (static_cast<int64_t>(layer) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (row & (G - 1));
    const uint32_t *q_row = reinterpret_cast<const uint32_t *>(q + at * D);
    float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
    for (int p = x.tile_begin * PASTA_TILE_PAGES; p < last; ++p) {
      const int page = plan[a.off_pages + x.page_off + p], meta = plan[a.off_pmeta + x.page_off + p];
      if (page < 0 || page >= pv.n_pages || meta < 0) continue;               // (reported when it was to be copied)
      const int sees = plan[a.off_vis + x.vis_off + thread * x.n_streams + min(PASTA_PMETA_STREAM(meta), x.n_streams - 1)] -
                       PASTA_PMETA_PAGE(meta) * PASTA_PAGE;
      if (sees <= 0) continue;
      const uint8_t *block = head + static_cast<int64_t>(page) * pv.n_kv_heads * BLOCK;
      float s = 0.f;
#pragma unroll 1
      for (int g = lane >> 4; g < D / kKv4Group; g += 2) {
        const uint4 c = *reinterpret_cast<const uint4 *>(block + g * 256 + r * 16);
        const uint32_t t = *reinterpret_cast<const uint16_t *>(block + kv4_k_scales(D) + (r * (D / kKv4Group) + g) * 2);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w}, t2 = t | (t << 16), c2 = kv4_offset_of(t2);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t k = kv4_value(kv4_pair(w[i >> 2], i & 3), t2, c2), qi = __ldg(q_row + g * 16 + i);
          s = fmaf(bf16_hi(k), bf16_hi(qi), fmaf(bf16_lo(k), bf16_lo(qi), s));
        }
      }
      s = __fmul_rn(s + __shfl_xor_sync(0xffffffffu, s, 16), a.scale_log2);
      if (kCap) s = softcap(s * a.cap_inv, pv.softcap_log2);
      if (r >= sees) s = -INFINITY;
      float top = s;
#pragma unroll
      for (int i = 8; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
      top = fmaxf(m, top);
      const float ref = top > -INFINITY ? top : 0.f;                           // (scores below the range of fp32 weigh nothing)
      float w = fast_exp2(__fadd_rn(s, -ref)), sum = w;
#pragma unroll
      for (int i = 8; i > 0; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
      const float before = l * fast_exp2(m - ref);
      m = top;
      l = before + sum;
      const float inv = l > 0.f ? 1.f / l : 0.f;
      w *= inv;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint2 c = *reinterpret_cast<const uint2 *>(block + kv4_v_codes(D) + (lane * E + e) * 8);
        o[e] *= before * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t t2 = *reinterpret_cast<const uint32_t *>(block + kv4_v_scales(D) + (lane * E / kKv4Group) * 32 + j * 4);
          const uint32_t v = kv4_value(kv4_pair(j < 4 ? c.x : c.y, j & 3), t2, kv4_offset_of(t2));
          o[e] = fmaf(__shfl_sync(0xffffffffu, w, 2 * j), bf16_lo(v), o[e]);
          o[e] = fmaf(__shfl_sync(0xffffffffu, w, 2 * j + 1), bf16_hi(v), o[e]);
        }
      }
    }
    if (l != l) {                                                              // a query that is not finite, or a score above the range of fp32
      m = not_a_row().x;
      l = not_a_row().y;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = NAN;
    }
    if (x.final_rows != 0) {
      if (a.lse && lane == 0) a.lse[at] = (m + log2f(l)) * 0.6931471805599453f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.out)[at * D + lane * E + e] = __float2bfloat16_rn(o[e]);
        else static_cast<float *>(a.out)[at * D + lane * E + e] = o[e];
      }
    } else {
      const int64_t part = static_cast<int64_t>(layer) * pv.rows_per_layer + x.row_base + row;
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(o[e]));
      if (warp_max(top) * l >= O_PART) {                                         // (l is at most 2^22: a run's tokens)
        m += 24.f;
        l *= 0x1p-24f;
      }
      if (lane == 0) pv.part_ml[part] = make_float2(m, l);
#pragma unroll
      for (int e = 0; e < E; ++e) pv.part_o[part * D + lane * E + e] = o[e] * l;
    }
  }
}

template <int D, int NMAX, bool kCap>
__global__ void __launch_bounds__(U<D, NMAX>::THREADS, U<D, NMAX>::RESIDENT)
attn_kv4_kernel(PoolView pv, TensorArgs a, const __nv_bfloat16 *__restrict__ q) {
  using L = U<D, NMAX>;
  constexpr int H = L::H;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t *sm = smem_raw + (base - raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = pv.n_q_heads / pv.n_kv_heads;
  const int g_shift = 31 - __clz(G);                              // G is 1, 2, 4 or 8
  const uint32_t bar = base + L::OFF_BAR;
  int32_t *meta_s = reinterpret_cast<int32_t *>(sm + L::OFF_META);
  uint32_t *misc = reinterpret_cast<uint32_t *>(sm + L::OFF_MISC);
  int32_t *unit_s = reinterpret_cast<int32_t *>(misc + 4);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(misc + 1);
  volatile int *far_flag = reinterpret_cast<volatile int *>(misc + 2);        // the unit is one for plain_rows
  float *ref_s = reinterpret_cast<float *>(sm + L::OFF_REF), *fact_s = reinterpret_cast<float *>(sm + L::OFF_FACT);
  float *warp_s = reinterpret_cast<float *>(sm + L::OFF_WARP);
  int32_t *row_s = reinterpret_cast<int32_t *>(warp_s);
  volatile uint32_t *seen_s = reinterpret_cast<volatile uint32_t *>(sm + L::OFF_SEEN), *saw_s = seen_s + 32, *waiting_s = seen_s + 64;
  // of threads 16 r to 16 r + 15 those that see their first tokens in this tile
  auto fresh = [&](int r) { return waiting_s[r] & (seen_s[r] | seen_s[8 + r] | seen_s[16 + r] | seen_s[24 + r]); };
  const int32_t *plan = pv.plan;

  if (tid == 0) {
    for (int b = 0; b < L::B_COUNT; ++b) mbar_init(bar + 8 * b, b == L::B_DRAIN ? 4 : 1);
    misc[1] = misc[2] = 0;
    unit_s[0] = -1;                                   // the last number taken
    mbar_init_fence();
  }
  fence_proxy_async();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::OFF_MISC), "r"(L::COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // no page is seen before a copy says so
  for (int i = tid; i < L::STAGES * PASTA_TILE_PAGES; i += L::THREADS) meta_s[i] = -1;
  // operand bytes that no copy fills meet zero weights, so they only have to be finite: page slots that a partial tile leaves empty
  for (int i = tid; i < L::STAGES * L::STAGE_BYTES / 16; i += L::THREADS) reinterpret_cast<uint4 *>(sm + L::OFF_STAGE)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  grid_dependency_wait();
  grid_launch_dependents();
  const long long limit = pv.wait_limit;
  int32_t *counter = pv.status + PASTA_STATUS_TAIL_COUNTER;
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  const int wq = warp & 3, half = warp >> 2;          // the quarter of TMEM this warp reaches, its part of the work
  const int token = wq * 32 + lane;                   // as a thread of the scores; as one of V and O: channel `token` (head_dim 64: % 64)
  const uint32_t lane_addr = tmem + (static_cast<uint32_t>(wq * 32) << 16);
  // the constants of kv4_pair in registers: as immediates they take two instructions instead of one
  uint32_t code_mask = 0x00780078u, code_one = 0x3f803f80u;
  asm volatile("" : "+r"(code_mask), "+r"(code_one));
  auto pair_of = [&](uint32_t w, int i) {
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(__funnelshift_r(w, w, 4 * i)), "r"(code_mask), "r"(code_one));
    return y;
  };
  const uint64_t scale2 = two_floats(a.scale_log2, a.scale_log2);
  const uint64_t q_desc = smem_desc(base + L::OFF_Q, 16, 1024);
  const uint64_t p_desc = L::NARROW ? smem_desc64(base + L::OFF_P, 512, L::P_GROUP) : smem_desc(base + L::OFF_P, 1024, L::P_GROUP);
  // test hook: held MMAs, so that what waits for them runs into its limit
  const bool no_mma = pv.debug_hold & 2;
  uint32_t it = 0, copied = 0;                        // tiles worked on (MMA phases follow it); tiles of the unit that were copied
  // (where nothing is assigned in advance, the first units go to the CTAs in order and the counter counts those behind them)
  const bool none_assigned = a.n_tunits == 0;
  int ll = none_assigned ? a.layer_count : -1, u = 0, u1 = 0, layer = 0, asked = 0;
  UnitInfo x;
  // The units assigned to the CTA in the next layer that has some.  A layer's ranges are taken by other CTAs than the layer's before:
  // what makes a range slow (masks, unit ends) is the same in every layer.
  auto next_range = [&]() {
    while (u == u1 && ++ll < a.layer_count) {
      const int range = (blockIdx.x + ll * (gridDim.x * 3 / 8 | 1)) % gridDim.x;
      u = plan[a.off_tcta + 2 * range];
      u1 = plan[a.off_tcta + 2 * range + 1];
    }
  };
  next_range();

  const int counted_from = none_assigned ? gridDim.x : 0, n_shared = a.n_dunits * a.layer_count;
  // The first thread takes numbers until one is past the last unit.  Every CTA ends with one such number, and the CTA that has the last
  // of them sets the counter back.  Nobody counts where the first units are all there are.
  const bool counted = a.n_dunits != 0 && n_shared > counted_from;
  auto take = [&]() {
    const int number = counted_from + atomicAdd(counter, 1);
    if (number == n_shared + static_cast<int>(gridDim.x) - 1) *counter = 0;
    unit_s[0] = number;
  };
  // ---- the next unit: those assigned to the CTA, layer by layer, then those handed out at run time (`taken`, from the counter)
  auto next_unit = [&](int taken) {
    int id = u, off = a.off_tunit;
    if (u < u1) {
      layer = ll;
      ++u;
      next_range();
    } else {
      if (taken >= n_shared) return false;
      id = taken / a.layer_count;
      layer = taken - id * a.layer_count;
      off = a.off_dunit;
    }
    x = load_unit(plan, off, 0, id);
    return true;
  };
  // Copies: every warp has PW pages of a tile, 16 bytes to a lane (bulk copies take 100 to 150 cycles each where eight leave together,
  // and the next barrier waits for the warps that issue them).  A lane holds a page's id and meta, asked for a tile ahead.
  constexpr int PW = PASTA_TILE_PAGES / (4 * H), PARTS = L::BLOCK / 16;
  int next_page = -1, next_meta = -1;                 // lane PW t + i: page i of the t-th tile asked for (-1: no page here)
  auto ask = [&](int count) {
    const int at = (x.tile_begin + asked + lane / PW) * PASTA_TILE_PAGES + warp * PW + lane % PW;
    next_page = next_meta = -1;
    if (lane < count * PW && at < x.n_pages) {
      next_page = plan[a.off_pages + x.page_off + at];
      next_meta = plan[a.off_pmeta + x.page_off + at];
    }
    asked += count;
  };
  auto copy = [&](int t) {
    const int s = copied % L::STAGES;
    if (lane / PW == t) {
      if (next_meta < 0 ? next_page != -1 : next_page < 0 || next_page >= pv.n_pages) {
        report(pv.status, PASTA_ERR_DEVICE_CHECK);
        next_page = next_meta = -1;
      }
      meta_s[s * PASTA_TILE_PAGES + warp * PW + lane % PW] = next_meta;
    }
    const uint8_t *head = pv.kv_base + (a.layer_begin + layer) * pv.layer_stride + static_cast<int64_t>(x.g) * L::BLOCK;
    const uint8_t *src[PW];
    bool there[PW];
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int page = __shfl_sync(0xffffffffu, next_page, PW * t + i);
      there[i] = page >= 0;
      src[i] = head + static_cast<int64_t>(page) * pv.n_kv_heads * L::BLOCK + (lane - i * PARTS) * 16;
    }
    const uint32_t dst = base + L::OFF_STAGE + s * L::STAGE_BYTES + warp * PW * L::BLOCK + lane * 16;
#pragma unroll
    for (int i = 0; i < (PW * PARTS + 31) / 32; ++i) {
      const bool second = PW == 2 && lane + 32 * i >= PARTS;
      if (lane + 32 * i < PW * PARTS && (second ? there[PW - 1] : there[0])) copy16(dst + i * 512, (second ? src[PW - 1] : src[0]) + i * 512, policy);
    }
    ++copied;
  };
  // a unit's first tiles; a group of copies per stage, empty where the unit has no tile for it
  auto first_pages = [&]() {
    asked = 0;
    copied = 0;
    ask(min(x.tile_end - x.tile_begin, L::STAGES));
  };
  auto first_copies = [&]() {
    const int nt = x.tile_end - x.tile_begin;
#pragma unroll 1
    for (int t = 0; t < L::STAGES; ++t) {
      if (t < nt) copy(t);
      copies_commit();
    }
    ask(asked < nt);
  };

  if (u == u1 && !none_assigned && counted) {
    if (tid == 0) take();
    __syncthreads();
  }
  bool more = next_unit(none_assigned ? blockIdx.x : counted ? unit_s[0] : n_shared);
  if (more) {
    first_pages();
    first_copies();
  }
  // A row's reference is 0 at first: weights are 2^score, scores above R_SLACK raise it, and a row whose sum shows that its scores
  // are far below (or all minus infinity) has its unit done again, carefully: first references from the first tokens' maxima.
  bool careful = false;
units:
  while (more) {
    if (careful && *far_flag != 0) break;                // to be done without tensor cores
    const int nt = x.tile_end - x.tile_begin;
    const int rows = x.n_threads << g_shift, n = (rows + 15) & ~15;
    const bool fin = x.final_rows != 0;

    // ---- stacked queries, four threads to a row; a row's first reference: NaN spoils a row whose query is not finite
    {
      constexpr int PER = D / 32;
      const int part = tid & 3;
#pragma unroll 1
      for (int row = tid >> 2; row < n; row += L::THREADS / 4) {
        uint4 val[PER];
#pragma unroll
        for (int c = 0; c < PER; ++c) val[c] = make_uint4(0, 0, 0, 0);
        if (row < rows) {
          const int qn = plan[a.off_tq + x.tq_off + (row >> g_shift)];
          const uint4 *src = reinterpret_cast<const uint4 *>(
              q + ((static_cast<int64_t>(layer) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (row & (G - 1))) * D) + part * PER;
#pragma unroll
          for (int c = 0; c < PER; ++c) val[c] = __ldg(src + c);
        }
        uint32_t m2 = 0;
#pragma unroll
        for (int c = 0; c < PER; ++c)
          m2 = __vmaxu2(__vmaxu2(m2, val[c].x & 0x7fff7fffu),
                        __vmaxu2(__vmaxu2(val[c].y & 0x7fff7fffu, val[c].z & 0x7fff7fffu), val[c].w & 0x7fff7fffu));
        m2 = __vmaxu2(m2, __shfl_xor_sync(0xfu << (lane & 28), m2, 1));
        m2 = __vmaxu2(m2, __shfl_xor_sync(0xfu << (lane & 28), m2, 2));
        if (part == 0) ref_s[row] = row >= rows ? 0.f : (m2 & 0xffffu) >= 0x7f80u || m2 >= 0x7f800000u ? NAN : careful ? R_UNSET : 0.f;
        uint8_t *dst = sm + L::OFF_Q + (row >> 3) * 1024 + (row & 7) * 128;
#pragma unroll
        for (int c = 0; c < PER; ++c) {
          const int chunk = part * PER + c;
          *reinterpret_cast<uint4 *>(dst + (chunk >> 3) * (NMAX * 128) + (((chunk & 7) ^ (row & 7)) << 4)) = val[c];
        }
      }
      fence_proxy_async();
    }
    if (tid < 8) waiting_s[tid] = tid * 16 >= x.n_threads ? 0 : 0xffffu >> max(0, 16 * tid + 16 - x.n_threads);
    if (tid >= 32 && tid < 64) saw_s[tid - 32] = 0;
    bool all_seen = !careful;
    copies_wait<L::STAGES - 1>();
    __syncthreads();
    float l[L::CHUNKS][8];
#pragma unroll
    for (int c = 0; c < L::CHUNKS; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) l[c][j] = 0.f;

    // How much of this token's page the request's threads see, 16 threads at a time, one to a lane of the half warp that has the page
    // (the first 32 threads are looked up a tile ahead); pages that every thread sees in full need no look.
    int meta = 0, visible_a = 0, visible_b = 0;
    bool masked = false, saw_all = false;
    auto visible = [&](int t0) {
      const int t = t0 + (lane & 15);
      if (meta < 0 || t >= x.n_threads) return 0;
      return plan[a.off_vis + x.vis_off + t * x.n_streams + min(PASTA_PMETA_STREAM(meta), x.n_streams - 1)] - PASTA_PMETA_PAGE(meta) * PASTA_PAGE;
    };
    auto look = [&](int s) {
      meta = meta_s[s * PASTA_TILE_PAGES + (token >> 4)];
      masked = __any_sync(0xffffffffu, meta < 0 || !(meta & PASTA_PMETA_ALL_VISIBLE));
      if (masked) {
        visible_a = visible(0);
        if (x.n_threads > 16) visible_b = visible(16);
      }
    };
    look(0);
    for (int k = 0; k < nt; ++k, ++it) {
      const int s = k % L::STAGES;
      const uint8_t *stage = sm + L::OFF_STAGE + s * L::STAGE_BYTES;
      // ---- K's codes to the A operand, a thread per token (half the channels); the P.V before has read what it replaces
      if (k > 0) cta_wait(bar + 8 * L::B_PV, (it - 1) & 1, abort_flag, limit);
      tc_fence_after();
      if (!all_seen && half == 0) {
        for (int r = 0; 16 * r < x.n_threads; ++r) {
          const uint32_t who = masked ? __ballot_sync(0xffffffffu, (r == 0 ? visible_a : r == 1 ? visible_b : visible(16 * r)) > 0) : 0xffffu;
          if (lane == 0) seen_s[8 * wq + r] = who | (who >> 16);
        }
      }
      {
        const uint8_t *block = stage + (token >> 4) * L::BLOCK;
        const uint8_t *at = block + (token & 15) * 16, *at_scale = block + kv4_k_scales(D) + (token & 15) * (D / 16);
        constexpr int GROUPS = (D / 32 + H - 1) / H;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
          const int g = half * GROUPS + i;
          if (GROUPS * H > D / 32 && g >= D / 32) break;
          const uint4 c = *reinterpret_cast<const uint4 *>(at + g * 256);
          const uint32_t t = *reinterpret_cast<const uint16_t *>(at_scale + 2 * g), t2 = t | (t << 16), c2 = kv4_offset_of(t2);
          const uint32_t w[4] = {c.x, c.y, c.z, c.w};
          uint32_t o[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = kv4_value(pair_of(w[e >> 2], e & 3), t2, c2);
          tmem_st16(lane_addr + L::COL_A + g * 16, o);
        }
      }
      tmem_st_wait();
      tc_fence_before();
      __syncthreads();
      if (warp == (it & 3) && !no_mma && elect_lane()) {
        // ---- S^T = K . Q^T
        tc_fence_after();
        const uint32_t idesc = IDESC4 | ((static_cast<uint32_t>(n) >> 3) << 17);
#pragma unroll
        for (int ks = 0; ks < L::KSTEPS; ++ks)
          mma_ts(tmem + L::COL_S, tmem + L::COL_A + ks * 8, q_desc + (((ks >> 2) * (NMAX * 128) + (ks & 3) * 32) >> 4), idesc, ks > 0);
        mma_commit(bar + 8 * L::B_QK);
      }
      __syncwarp();
      bool first = false;
      if (!all_seen) {
        all_seen = true;
        for (int r = 0; 16 * r < x.n_threads; ++r) {
          const uint32_t f = fresh(r);
          first |= f != 0;
          all_seen &= waiting_s[r] == f;
        }
      }
      // ---- which threads of the request see this token, a bit each: most see all or nothing of a page, the others are gone through
      constexpr int WORDS = (NMAX + 31) / 32;
      uint32_t seen[WORDS];
      if (masked) {
#pragma unroll
        for (int r = 0; r < 2 * WORDS; ++r) {
          if (r % 2 == 0) seen[r / 2] = 0;
          if (16 * r >= x.n_threads) continue;
          const int v = r == 0 ? visible_a : r == 1 ? visible_b : visible(16 * r);
          uint32_t who = __ballot_sync(0xffffffffu, v >= PASTA_PAGE);
          uint32_t some = __ballot_sync(0xffffffffu, v > 0 && v < PASTA_PAGE);
          some |= some >> 16;
          if (half == 0 && lane == 0) saw_s[8 * wq + r] |= who | (who >> 16) | some;
          who >>= lane & 16;
          for (; some & 0xffffu; some &= some - 1) {
            const int j = __ffs(some) - 1;
            if ((lane & 15) < __shfl_sync(0xffffffffu, v, (lane & 16) | j)) who |= 1u << j;
          }
          seen[r / 2] |= (who & 0xffffu) << (16 * (r % 2));
        }
      } else {
        saw_all = true;
      }
      // (a unit's last tile: the unit behind it, if it is one of those handed out at run time, while the scores are worked out)
      if (k + 1 == nt && tid == 0 && counted && u == u1 && !careful) take();
      cta_wait(bar + 8 * L::B_QK, it & 1, abort_flag, limit);
      tc_fence_after();
      // ---- V's codes to the A operand, in K's place, a thread per channel (half the pages)
      {
        const int channel = token % D;
        constexpr int PAGES = L::VSTEPS / H;
        const int page0 = (D == 128 ? 0 : 4 * (wq >> 1)) + half * PAGES;
        const uint8_t *at = stage + page0 * L::BLOCK + kv4_v_codes(D) + channel * 8;
        const uint8_t *at_scale = stage + page0 * L::BLOCK + kv4_v_scales(D) + (channel / kKv4Group) * 32;
#pragma unroll
        for (int p = 0; p < PAGES; ++p) {
          const uint2 c = *reinterpret_cast<const uint2 *>(at + p * L::BLOCK);
          const uint4 ta = *reinterpret_cast<const uint4 *>(at_scale + p * L::BLOCK), tb = *reinterpret_cast<const uint4 *>(at_scale + p * L::BLOCK + 16);
          const uint32_t t[8] = {ta.x, ta.y, ta.z, ta.w, tb.x, tb.y, tb.z, tb.w};
          uint32_t o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = kv4_value(pair_of(i < 4 ? c.x : c.y, i & 3), t[i], kv4_offset_of(t[i]));
          tmem_st8(lane_addr + L::COL_A + (half * PAGES + p) * 8, o);
        }
      }
      // ---- the tile's weights
      auto hide = [&](int c, float *v) {            // c: chunk of rows
        const int t0 = 8 * c >> g_shift;
        uint32_t w = seen[0];
#pragma unroll
        for (int i = 1; i < WORDS; ++i) w = (t0 >> 5) == i ? seen[i] : w;
        w >>= t0 & 31;
        if (g_shift >= 2) {
          const bool low = w & 1, high = w & (g_shift == 2 ? 2 : 1);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (j < 4 ? low : high) ? v[j] : -INFINITY;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (w >> (j >> g_shift)) & 1 ? v[j] : -INFINITY;
        }
      };
      // scores of chunk c as they come from the MMA; scaled (log2 units), capped and masked; and relative to the references
      auto scores = [&](int c, float *v) { tmem_ld8_issue(lane_addr + L::COL_S + c * 8, reinterpret_cast<uint32_t *>(v)); };
      auto finish = [&](int c, float *v, auto hidden) {
        if (kCap) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= a.scale_log2 * a.cap_inv;
          softcap_columns<8>(v, pv.softcap_log2, true);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= a.scale_log2;
        }
        if (decltype(hidden)::value) hide(c, v);
      };
      auto relative = [&](int c, float *v, auto hidden) {
        const float4 r0 = *reinterpret_cast<const float4 *>(ref_s + c * 8), r1 = *reinterpret_cast<const float4 *>(ref_s + c * 8 + 4);
        if (kCap) {
          finish(c, v, hidden);
          v[0] += r0.x; v[1] += r0.y; v[2] += r0.z; v[3] += r0.w; v[4] += r1.x; v[5] += r1.y; v[6] += r1.z; v[7] += r1.w;
        } else {
          fma2s(v[0], v[1], scale2, r0.x, r0.y);
          fma2s(v[2], v[3], scale2, r0.z, r0.w);
          fma2s(v[4], v[5], scale2, r1.x, r1.y);
          fma2s(v[6], v[7], scale2, r1.z, r1.w);
          if (decltype(hidden)::value) hide(c, v);
        }
      };
      // this token's row of the B operand: its 16-byte chunk x is at x ^ (row % 8) (or ^ (row / 2 % 4) in rows of 64 bytes), and at
      // head_dim 64 the two halves of the tile have every other chunk
      const int b_row = D == 128 ? token : token & 63, b_half = D == 128 ? 0 : token >> 6;
      const uint32_t p_row = L::NARROW
          ? L::OFF_P + (b_row >> 3) * L::P_GROUP + (b_row & 7) * 64 + ((((b_row >> 1) & 3) ^ b_half) << 4)
          : L::OFF_P + (b_row >> 3) * L::P_GROUP + (b_row & 7) * 128 + (((b_row & 7) ^ b_half) << 4);
      auto place = [&](int c) {
        const int col = L::OW * c;
        if (L::NARROW) return reinterpret_cast<uint4 *>(sm + (p_row ^ ((col & 3) << 4)));
        return reinterpret_cast<uint4 *>(sm + (p_row ^ ((col & 7) << 4)) + (col >> 3) * 1024);
      };
      // Weights rounded to bf16, as rows of the B operand; returns the largest exponent.  Straight code for every number of chunks
      // (rows beyond the unit's last are zeros in Q and count for nothing): a branch costs as much as half a chunk, and chunks overlap.
      // Capped scores take so much code that fetching it costs more than that: a loop over the chunks.
      auto chunk_weights = [&](int c, float *y, float &top, uint32_t *o, auto hidden) {
        relative(c, y, hidden);
        top = max3(max3(top, y[0], y[1]), y[2], y[3]);
        top = max3(max3(top, y[4], y[5]), y[6], y[7]);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pack_bf16(fast_exp2(y[2 * j]), fast_exp2(y[2 * j + 1]));
        *place(c) = make_uint4(o[0], o[1], o[2], o[3]);
      };
      auto weights = [&](auto chunks, auto hidden) {
        constexpr int C = decltype(chunks)::value;
        float top = -INFINITY;
        uint32_t o[4];
#pragma unroll
        for (int c0 = 0; c0 < C; c0 += 4) {
          float v[4][8];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c0 + i < C) scores(H * (c0 + i) + half, v[i]);
          tmem_ld_wait8(reinterpret_cast<uint32_t *>(v[0]));
#pragma unroll
          for (int i = 1; i < 4; ++i)
            if (c0 + i < C) tmem_ld_order8(reinterpret_cast<uint32_t *>(v[i]));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c0 + i < C) chunk_weights(H * (c0 + i) + half, v[i], top, o, hidden);
        }
        return top;
      };
      const int my_chunks = ((n >> 3) - half + H - 1) / H;
      auto by_chunks = [&](auto f) {                // f for the number of chunks of this thread
#define PASTA_C(cc) \
  if constexpr (L::CHUNKS >= cc && cc * H % 2 == 0) { if (my_chunks == cc) return f(std::integral_constant<int, cc>()); }
        PASTA_C(1) PASTA_C(2) PASTA_C(3) PASTA_C(4) PASTA_C(5)
#undef PASTA_C
        return -INFINITY;
      };
      auto all_weights = [&]() {
        if constexpr (kCap) {
          float top = -INFINITY;
#pragma unroll 1
          for (int c = half; 8 * c < n; c += H) {
            float y[8];
            uint32_t o[4];
            scores(c, y);
            tmem_ld_wait8(reinterpret_cast<uint32_t *>(y));
            if (masked) chunk_weights(c, y, top, o, std::true_type());
            else chunk_weights(c, y, top, o, std::false_type());
          }
          return top;
        } else {
          return by_chunks([&](auto chunks) { return masked ? weights(chunks, std::true_type()) : weights(chunks, std::false_type()); });
        }
      };
      // maxima of the rows of a chunk over the warp's tokens
      auto maxima = [&](int c) {
        float y[8], mine = -INFINITY;
        scores(c, y);
        tmem_ld_wait8(reinterpret_cast<uint32_t *>(y));
        if (masked) finish(c, y, std::true_type());
        else finish(c, y, std::false_type());
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float m = warp_max(y[j]);
          if (lane == j) mine = m;
        }
        if (lane < 8) warp_s[wq * NMAX + 8 * c + lane] = mine;
      };
      auto maximum = [&]() { return fmaxf(fmaxf(warp_s[tid], warp_s[NMAX + tid]), fmaxf(warp_s[2 * NMAX + tid], warp_s[3 * NMAX + tid])); };
      if (first) {
        // ---- rows that see their first tokens get their references before any weight is worked out (their O and l are zero)
#pragma unroll 1
        for (int c = half; 8 * c < rows; c += H) {
          const int t0 = 8 * c >> g_shift, t1 = (8 * c + 7) >> g_shift;
          if (fresh(t0 >> 4) & ((2u << (t1 & 15)) - (1u << (t0 & 15)))) maxima(c);
        }
        __syncthreads();
        if (tid < rows && ((fresh(tid >> g_shift >> 4) >> (tid >> g_shift & 15)) & 1) && ref_s[tid] == R_UNSET) {
          const float m = maximum();
          if (m > -INFINITY) ref_s[tid] = -m;
        }
        __syncthreads();
        if (tid < 8) waiting_s[tid] &= ~fresh(tid);
      }
      bool raised = false, left = false;
      for (;;) {
        const float top = all_weights();
        copies_wait<L::STAGES - 2>();                // the next tile's
        tmem_st_wait();
        fence_proxy_async();
        tc_fence_before();
        // ---- everybody is done with the stage, V's operand and the weights stand, and the CTA votes (also on leaving)
        if (!__syncthreads_or((!raised && top > R_SLACK) || *abort_flag != 0)) break;
        left = __syncthreads_or(*abort_flag != 0);
        if (left) break;
        // ---- some row's reference goes up: maxima of all rows over the tile, then O and l brought to the new references
#pragma unroll 1
        for (int c = half; 8 * c < rows; c += H) maxima(c);
        __syncthreads();
        if (tid < n) {
          float f = 1.f;
          if (tid < rows) {
            const float m = maximum();
            const float old = ref_s[tid];
            if (m > -INFINITY && (old == R_UNSET || m + old > R_SLACK)) {
              f = old == R_UNSET ? 0.f : fast_exp2(-old - m);          // (a row that has seen nothing has nothing to bring along)
              ref_s[tid] = -m;
            }
          }
          fact_s[tid] = f;
        }
        __syncthreads();
        if (k > 0) {                                 // (the P.V before has finished: it was waited for)
#pragma unroll
          for (int i = 0; i < L::CHUNKS; ++i) {
            const int c = H * i + half;
            if (8 * c >= rows) continue;
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              f[j] = fact_s[8 * c + j];
              l[i][j] *= f[j];
            }
#pragma unroll 1
            for (int o2 = 0; o2 < L::OW; ++o2) {
              uint32_t o[8];
              const uint32_t at = lane_addr + L::COL_O + 8 * (L::OW * c + o2);
              tmem_ld8_issue(at, o);
              tmem_ld_wait8(o);
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f[j]);
              tmem_st8(at, o);
            }
          }
          tmem_st_wait();
        }
        raised = true;
      }
      if (left) break;
      if (k + L::STAGES < nt) {
        copy(0);
        ask(asked < nt);
      }
      copies_commit();
      if (warp == ((it + 2) & 3) && !no_mma && elect_lane()) {
        // ---- O^T += V^T . P^T
        tc_fence_after();
        const uint32_t idesc = IDESC4_PV | (((L::OW * static_cast<uint32_t>(n)) >> 3) << 17);
#pragma unroll
        for (int ks = 0; ks < L::VSTEPS; ++ks)
          mma_ts(tmem + L::COL_O, tmem + L::COL_A + ks * 8, p_desc + (ks * 2 * L::P_GROUP >> 4), idesc, k > 0 || ks > 0);
        mma_commit(bar + 8 * L::B_PV);
      }
      __syncwarp();
      // ---- the sums, of the weights as rounded
#pragma unroll
      for (int i = 0; i < L::CHUNKS; ++i) {
        if (8 * (H * i + half) >= n) continue;
        const uint4 w = *place(H * i + half);
        const uint32_t o[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) add_bf16x2(l[i][2 * j], l[i][2 * j + 1], o[j]);
      }
      if (k + 1 < nt) look((k + 1) % L::STAGES);
    }
    if (saw_all && half == 0 && lane < 8) saw_s[8 * wq + lane] = 0xffffu;
    if (__syncthreads_or(*abort_flag != 0)) break;

    // ---- epilogue: sums over the tokens, then the rows of O, a thread per channel
#pragma unroll
    for (int i = 0; i < L::CHUNKS; ++i) {
      const int c = H * i + half;
      if (8 * c >= rows) continue;
      const float t = warp_sum8(l[i], lane);
      if ((lane & 3) == 0) warp_s[wq * NMAX + 8 * c + (lane >> 2)] = t;
    }
    __syncthreads();
    bool faint = false, look_at_o = false, small = false;
    int32_t *top_s = reinterpret_cast<int32_t *>(warp_s) + NMAX;       // [NMAX] largest magnitude in a row of O (where the thread has read its row's sums)
    if (tid < rows) {
      const float sum = (warp_s[tid] + warp_s[NMAX + tid]) + (warp_s[2 * NMAX + tid] + warp_s[3 * NMAX + tid]);
      const bool spoilt = sum != sum;
      const float m = spoilt ? not_a_row().x : sum > 0.f ? -ref_s[tid] : -INFINITY, l_all = spoilt ? not_a_row().y : sum;
      fact_s[tid] = spoilt ? NAN : fin ? (sum > 0.f ? 1.f / sum : 0.f) : 1.f;
      int at;                                          // the row's place among all rows of its kind
      if (fin) {
        at = (layer * a.n_queries + plan[a.off_tq + x.tq_off + (tid >> g_shift)]) * pv.n_q_heads + x.g * G + (tid & (G - 1));
        if (a.lse) a.lse[at] = (m + log2f(l_all)) * 0.6931471805599453f;
      } else {
        at = layer * pv.rows_per_layer + x.row_base + tid;
        pv.part_ml[at] = make_float2(m, l_all);
      }
      const int thread = tid >> g_shift;
      const uint32_t saw = saw_s[thread >> 4] | saw_s[8 + (thread >> 4)] | saw_s[16 + (thread >> 4)] | saw_s[24 + (thread >> 4)];
      faint = !careful && sum < R_FAINT && ((saw >> (thread & 15)) & 1);
      if (!kCap && is_far(ref_s[tid])) {
        faint = true;
        *far_flag = 1;
      }
      small = !careful && sum > 0.f && sum < L_TINY;
      look_at_o = small || sum > (fin ? L_FINAL : L_PART);
      top_s[tid] = 0;
      row_s[tid] = at;                                 // (where the thread has read its row's first sum)
    }
    cta_wait(bar + 8 * L::B_PV, (it - 1) & 1, abort_flag, limit);
    bool again = __syncthreads_or(faint || look_at_o || *abort_flag != 0);
    if (again && __syncthreads_or(*abort_flag != 0)) break;
    tc_fence_after();
    const uint32_t o_addr = lane_addr + L::COL_O + (D == 64 ? (wq >> 1) * 8 : 0);
    if (again) {
#pragma unroll 1
      for (int c = half; 8 * c < rows; c += H) {
        uint32_t o[8], mine = 0;
        tmem_ld8_issue(o_addr + c * 8 * L::OW, o);
        tmem_ld_wait8(o);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t top = __reduce_max_sync(0xffffffffu, o[j] & 0x7fffffffu);
          if (lane == j) mine = top;
        }
        if (lane < 8 && 8 * c + lane < rows) atomicMax(top_s + 8 * c + lane, static_cast<int>(mine));
      }
      __syncthreads();
      if (tid < rows && look_at_o) {
        const float top = __int_as_float(top_s[tid]);
        if (!(top < (fin ? INFINITY : O_PART))) {
          faint = true;
          *far_flag = 1;
        }
        faint |= small && top < O_TINY;
      }
      again = __syncthreads_or(faint);
    }
    // ---- the copies of the unit behind it, under way while this one's rows are written
    const int taken = counted ? unit_s[0] : n_shared;
    if (again) careful = true;
    else {
      careful = false;
      more = next_unit(taken);
    }
    if (more) {
      first_pages();
      first_copies();
    }
    if (again) continue;
    float *sum_s = reinterpret_cast<float *>(sm + L::OFF_P) + (token & 63);
    if constexpr (D == 64) {
      if (wq >= 2) {
#pragma unroll 1
        for (int c = half; 8 * c < rows; c += H) {
          uint32_t o[8];
          tmem_ld8_issue(o_addr + c * 8 * L::OW, o);
          tmem_ld_wait8(o);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum_s[(c * 8 + j) * 64] = __uint_as_float(o[j]);
        }
      }
      __syncthreads();
    }
    if (D == 128 || wq < 2) {
#pragma unroll 1
      for (int c = half; 8 * c < rows; c += H) {
        uint32_t o[8];
        tmem_ld8_issue(o_addr + c * 8 * L::OW, o);
        tmem_ld_wait8(o);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int row = c * 8 + j;
          if (row >= rows) continue;
          const float f = fact_s[row];
          float y = __uint_as_float(o[j]);
          if (D == 64) y += sum_s[row * 64];
          y = f == 0.f ? 0.f : y * f;                // a final row that saw nothing is written as zeros
          const int64_t at = static_cast<int64_t>(row_s[row]) * D + token;
          if (!fin) pv.part_o[at] = y;
          else if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
          else static_cast<float *>(a.out)[at] = y;
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  }

  if (more && *abort_flag == 0) {
    // ---- a unit with a row that is too far from 0, or too large (out here its code costs the units of the loop no registers)
    plain_rows<D, L::THREADS / 32, kCap>(pv, a, q, x, layer);
    copies_wait<0>();
    __syncthreads();
    if (tid == 0) *far_flag = 0;
    careful = false;
    more = next_unit(counted ? unit_s[0] : n_shared);
    if (more) {
      first_pages();
      first_copies();
    }
    __syncthreads();
    goto units;
  }

  // ---- tear-down
  copies_wait<0>();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // Some wait has run out and the whole CTA has left in the middle of its work: MMAs in flight end on their own and are waited for.
    // A commit follows the MMAs of the thread that makes it, so the lane that is elected to issue them makes it.
    if (warp < 4 && elect_lane()) {                    // every warp that issues MMAs
      mma_commit(bar + 8 * L::B_DRAIN);
      mbar_wait_bounded(bar + 8 * L::B_DRAIN, 0);
    }
    if (tid == 0) {
      while (counted && unit_s[0] < n_shared) take();
      report(pv.status, PASTA_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
  }
  if (warp == 0) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::COLS) : "memory");
  }
}

template <int D, int NMAX>
cudaError_t launch_t(const PoolView &pv, const PlanHeader &h, const TensorArgs &a, const void *q, cudaStream_t st) {
  using L = U<D, NMAX>;
  static uint64_t prepared[2] = {0, 0};
  const bool cap = pv.softcap_log2 > 0.f;
  const auto kernel = cap ? attn_kv4_kernel<D, NMAX, true> : attn_kv4_kernel<D, NMAX, false>;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void *>(kernel), L::SMEM_BYTES, &prepared[cap]);
  if (e != cudaSuccess) return e;
  const int grid = a.n_tunits ? h.w[PH_T_GRID] : static_cast<int>(std::min<int64_t>(h.w[PH_T_GRID], int64_t(a.n_dunits) * a.layer_count));
  return launch_overlapped(kernel, dim3(grid), dim3(L::THREADS), L::SMEM_BYTES, st, pv, a, static_cast<const __nv_bfloat16 *>(q));
}

template <int D>
cudaError_t launch_d(const PoolView &pv, const PlanHeader &h, const TensorArgs &a, const void *q, cudaStream_t st) {
  const int rows = h.w[PH_T_MAX_ROWS];
  constexpr int MOST = kv4_max_rows(D);
  static_assert(U<D, 32>::RESIDENT == kv4_ctas_per_sm(32) && U<D, MOST>::RESIDENT == kv4_ctas_per_sm(MOST), "the planner counts on it");
  const auto launch = rows <= 32 ? launch_t<D, 32> : launch_t<D, MOST>;
  return launch(pv, h, a, q, st);
}

}  // namespace

cudaError_t launch_attn_kv4(const PoolView &pv, const PlanHeader &h, int32_t layer_begin, int32_t layer_count,
                            const void *q, float scale_log2, void *out, float *lse, bool out_bf16, cudaStream_t st) {
  if (h.w[PH_T_GRID] == 0 || layer_count == 0) return cudaSuccess;
  TensorArgs a;
  a.off_tunit = h.w[PH_OFF_TUNIT]; a.off_treq = h.w[PH_OFF_TREQ]; a.off_tcta = h.w[PH_OFF_TCTA];
  a.off_pages = h.w[PH_OFF_PAGES]; a.off_pmeta = h.w[PH_OFF_PMETA]; a.off_vis = h.w[PH_OFF_VIS];
  a.off_tq = h.w[PH_OFF_TQ];
  a.off_dunit = h.w[PH_OFF_DUNIT]; a.n_dunits = h.w[PH_N_DUNITS]; a.n_tunits = h.w[PH_N_TUNITS];
  a.n_queries = h.w[PH_N_QUERIES]; a.layer_begin = layer_begin; a.layer_count = layer_count;
  a.scale_log2 = scale_log2;
  a.cap_inv = pv.softcap_log2 > 0.f ? 1.f / pv.softcap_log2 : 0.f;
  a.out = out; a.lse = lse; a.out_bf16 = out_bf16 ? 1 : 0;
  return pv.head_dim == 128 ? launch_d<128>(pv, h, a, q, st) : launch_d<64>(pv, h, a, q, st);
}

}  // namespace pasta
