// K2 of an 8-bit pool, head_dim 128: tensor-core pass over e4m3 codes (the plan, units and rows are those of attn_tensor.cu).
//
//   S[128 x 128] = (Qhi + Qlo)[128 x 128] . Kcodes^T   tcgen05.mma kind::f8f6f4 (N = 128, K = 32), operands from shared memory
//   p'           = 2^(S * factor * 2^ek + ev - ref)     factor: scale * log2e / the row's own scale; capped if asked for
//   O[128 x 128] += (P'0 + P'1 + P'2)[128 x 128] . Vcodes   tcgen05.mma, P' read from TMEM as the A operand
//   l            += p' 2^-ev                            out = O / l
//
// K's and V's codes are MMA operands as they lie in the page (128-byte rows with the 128-byte swizzle: K K-major, V MN-major);
// the page's scales enter where scores are turned into weights: ek in the factor, ev as an addend of the exponent, so that
// p' is the size of a token's contribution.  Eight bits are too few for queries and weights, so each is a sum of terms.
// A query is two e4m3 terms, hi and the rest: 8 significant bits, as many as bf16 has.  A query row is first scaled by a power
// of two that brings its largest magnitude to [2^7, 2^8): the split is exact down to 2^-10 of that and off by at most 2^-17 of
// it below.  A weight is three e5m2 terms.  A row may hold one large weight and thousands of small ones that are most of its
// result, so a weight needs range as well as bits, and e4m3's steps end at 2^-9 (two e4m3 terms lost up to a third of the output
// row behind one token of 0.9 of the weight and 32768 others).  An e5m2 code is the upper byte of an fp16 number, so the terms
// are bytes of the fp16 weight, of what is left of it, and of what is left then, rounded (split4): 9 significant bits, with no
// conversion but the one to fp16; the last rounding goes up in even columns and down in odd ones where it is a tie.
// The reference of a row is set 2^8 below its largest p' and raised when exceeded by more than 2^15, so a weight is off by at
// most 2^-8 of itself or 2^-24 of the row's largest contribution; l sums unrounded weights in fp32.
//
// What bounds it.  A tile of 128 tokens is 32 KB, 1408 cycles of the measured copy bandwidth per SM.  The MMAs take 1280
// (512 for two terms of queries, 768 for three of weights), during which they read shared memory at 64 to 128 bytes per cycle.
// The other half is the softmax, where every instruction of a warp costs the same for 4 rows as for 32 and a column of scores some
// 12 cycles of its scheduler, so with few rows they are put to use several times (NC columns per thread of the 64 of its half
// tile):
//   up to 32 rows  NC = 16: every TMEM quarter (32 lanes) holds a copy of the rows and answers for a quarter of the columns,
//   up to 64 rows  NC = 32: every pair of quarters holds a copy and answers for half of them,
//   more           NC = 64: one copy.
// A copy's weights for columns it does not answer for are zeros.  The two halves of a tile belong to two softmax groups, as in
// attn_tensor.cu; each copy of a row in each group has its own reference, sum and accumulator row, so nothing is exchanged
// between the softmax warps until the unit's epilogue.  Measured (us; one softmax thread per row and half tile throughout in
// brackets): 64 requests of 4 to 36 rows 180 (200), short capped responses 170 (229); 68 rows behind long prefixes 230.  The bf16
// pool takes 183, 189 and 234 for the same steps: the codes halve the bytes, and the instructions that replace them take as long.
//
// Warp roles (384 threads): warp 0 producer (4 or 5 stages of one tile), warp 1 MMA issue (one thread; Q.K^T runs one tile ahead
// of P.V, two score buffers in TMEM), warps 2-3 build the Q operand, warps 4-7 and 8-11 the two softmax groups.  Every wait is
// bounded; on expiry the CTA reports PASTA_ERR_TIMEOUT, drains and leaves.  (All lanes of a warp poll: with one
// lane that polls and tells the others the three cases took 8, 15 and 3 % longer.)
#include <cuda_fp16.h>

#include "tensor_common.cuh"

namespace pasta {

namespace {

constexpr int F_THREADS = 384;
constexpr int F_WARPS = 8;                                      // softmax: two groups of four warps
constexpr int F_HALF = T_TILE / 2;                              // columns of one softmax group
constexpr int F_FACTORS = 4;                                    // units whose rows' score factors are kept
constexpr int F_BLOCK = kv8_block_bytes(128);
constexpr int F_STAGE_BYTES = PASTA_TILE_PAGES * F_BLOCK;       // 32 KB
constexpr int F_Q_TERM = 128 * 128, F_Q_BYTES = 2 * F_Q_TERM;   // 32 KB: two terms
constexpr int F_SUM_BYTES = 16384;                              // per group: where the copies' accumulators are added up

// Shared memory and barriers (8 bytes each).  The room that copies' accumulators take to be added up is a stage's.
template <int NC>
struct F {
  static constexpr int STAGES = NC < 64 ? 4 : 5;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_STAGE = OFF_Q + F_Q_BYTES;
  static constexpr int OFF_SUM = OFF_STAGE + STAGES * F_STAGE_BYTES;
  static constexpr int OFF_BAR = OFF_SUM + (NC < 64 ? 2 * F_SUM_BYTES : 0);
// barriers (8 bytes each)
  static constexpr int B_FULL = 0, B_EMPTY = B_FULL + STAGES, B_SFULL = B_EMPTY + STAGES, B_PFULL = B_SFULL + 2,      // PFULL[2 b + group]
                B_QFULL = B_PFULL + 4, B_QFREE = B_QFULL + 1, B_OFULL = B_QFREE + 1, B_OFREE = B_OFULL + 1,
                B_MLFULL = B_OFREE + 1, B_SUM = B_MLFULL + 1,     // [group] the epilogue's additions
                B_FACTORS = B_SUM + 2,                            // the rows' score factors of unit uc % F_FACTORS are there
                B_DRAIN = B_FACTORS + F_FACTORS,                  // only used when a role gave up
                B_COUNT = B_DRAIN + 1;
  static constexpr int OFF_META = OFF_BAR + 8 * ((B_COUNT + 1) & ~1);    // per stage: 8 page metas
  static constexpr int OFF_SCALE = OFF_META + STAGES * 32;             // per stage: 8 pages' exponents, ek + (ev << 8)
  static constexpr int OFF_MISC = OFF_SCALE + STAGES * 32;             // tmem base, abort flag, shared units taken, their records
  static constexpr int OFF_ML = OFF_MISC + 16 + 64 * T_RING;             // [unit parity][warp][lane] (reference, sum) for the epilogue
  static constexpr int OFF_FACTORS = OFF_ML + 2 * F_WARPS * 256;         // [F_FACTORS][128] floats
  static constexpr int SMEM_BYTES = OFF_FACTORS + F_FACTORS * 512 + 1024;      // slack to align the base to 1024
  static_assert(OFF_META % 16 == 0 && OFF_MISC % 16 == 0, "records are read as int4");
  static_assert(SMEM_BYTES <= 232448, "shared memory budget");
};

// TMEM columns: S[b] at 128 b (group g's half at 64 g, its P in the first 48 of that: three terms of 16), O_g at 256 + 128 g
constexpr uint32_t COL_S = 0, COL_O = 256;
// D fp32, N = 128; A and B e4m3, or A e5m2 and B (= V) MN-major
constexpr uint32_t IDESC_QK8 = (1u << 4) | ((128u >> 3) << 17), IDESC_PV8 = IDESC_QK8 | (1u << 7) | (1u << 16);
constexpr float FAR_SCORE = 1048576.f;                          // log2 units: fp32 steps are 2^-3 there
constexpr float P_TOP = 8.f, P_SLACK = 15.f;                    // log2 of a row's largest p' when its reference is set, and at most

__device__ __forceinline__ void mma8_ss(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A operand from TMEM: row m in its lane, four codes per 32-bit column (32 K-elements = 8 columns)
__device__ __forceinline__ void mma8_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%4], {%0,%1,%2,%3};" ::"r"(a), "r"(b), "r"(c), "r"(d), "r"(taddr) : "memory");
}
// 16 consecutive columns of this thread's TMEM lane, waited for
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r) {
  tmem_ld16_issue(taddr, r);
  asm volatile("tcgen05.wait::ld.sync.aligned;" : PASTA_RW16(r) :: "memory");
}
// rows of a unit's MMAs: 64 when that holds the unit's rows in all copies (row i is then in lane 32 (i / 16) + i % 16: 16 to a
// quarter), else 128
template <int NC>
__device__ __forceinline__ bool unit_m64(int rows) { return NC == 16 ? rows <= 16 : NC == 64 ? rows <= 64 : false; }

// Four query elements as the e4m3 terms hi and lo (hi + lo = the number to 8 significant bits, in steps of 2^-9 at the least).
__device__ __forceinline__ void split_query4(float a, float b, float c, float d, uint32_t &hi, uint32_t &lo) {
  uint16_t h0, h1, l0, l1;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h0) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h1) : "f"(d), "f"(c));
  const uint32_t f0 = e4m3x2_to_f16x2(h0), f1 = e4m3x2_to_f16x2(h1);
  const __half2 g0 = __hsub2(__floats2half2_rn(a, b), *reinterpret_cast<const __half2 *>(&f0));
  const __half2 g1 = __hsub2(__floats2half2_rn(c, d), *reinterpret_cast<const __half2 *>(&f1));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l0) : "r"(*reinterpret_cast<const uint32_t *>(&g0)));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(l1) : "r"(*reinterpret_cast<const uint32_t *>(&g1)));
  hi = h0 | (static_cast<uint32_t>(h1) << 16);
  lo = l0 | (static_cast<uint32_t>(l1) << 16);
}

// Four weights, 0 <= p <= 2^15, as three e5m2 terms each: off by at most 2^-8 p, or 1.25 * 2^-17 where that is more
// (over all fp16 numbers; a NaN stays one).
__device__ __forceinline__ void split4(float a, float b, float c, float d, uint32_t *t) {
  auto rest = [](uint32_t h) {                    // what the upper bytes of two fp16 leave: exact
    const uint32_t top = h & 0xff00ff00u;
    const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&h), *reinterpret_cast<const __half2 *>(&top));
    return *reinterpret_cast<const uint32_t *>(&r);
  };
  uint32_t x, y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(b), "f"(a));
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(d), "f"(c));
  t[0] = __byte_perm(x, y, 0x7531);
  x = rest(x);
  y = rest(y);
  t[1] = __byte_perm(x, y, 0x7531);
  t[2] = __byte_perm(rest(x) + 0x007f0080u, rest(y) + 0x007f0080u, 0x7531);
}

// NC: columns per softmax thread: 16 when every unit of the plan has at most 32 rows, 32 up to 64, 64 otherwise
template <int NC, bool kCap>
__global__ void __launch_bounds__(F_THREADS, 1)
attn_kv8_tensor_kernel(PoolView pv, TensorArgs a, const __nv_bfloat16 *__restrict__ q) {
  using L = F<NC>;
  constexpr int F_STAGES = L::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t *sm = smem_raw + (base - raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = pv.n_q_heads / pv.n_kv_heads;
  const int g_shift = 31 - __clz(G);                              // G is 1, 2, 4 or 8
  const uint32_t bar = base + L::OFF_BAR;
  int32_t *meta_s = reinterpret_cast<int32_t *>(sm + L::OFF_META);
  int32_t *scale_s = reinterpret_cast<int32_t *>(sm + L::OFF_SCALE);
  uint32_t *misc = reinterpret_cast<uint32_t *>(sm + L::OFF_MISC);
  float *factor_s = reinterpret_cast<float *>(sm + L::OFF_FACTORS);
  float2 *ml_s = reinterpret_cast<float2 *>(sm + L::OFF_ML);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(misc + 1);
  const int32_t *plan = pv.plan;

  // ---- set-up (operand bytes that no copy fills meet zero weights, so they only have to be finite: see attn_tensor.cu)
  if (tid == 0) {
    for (int s = 0; s < F_STAGES; ++s) { mbar_init(bar + 8 * (L::B_FULL + s), 2); mbar_init(bar + 8 * (L::B_EMPTY + s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar + 8 * (L::B_SFULL + b), 1); mbar_init(bar + 8 * (L::B_SUM + b), 4); }
    for (int b = 0; b < 4; ++b) mbar_init(bar + 8 * (L::B_PFULL + b), 4);
    mbar_init(bar + 8 * L::B_QFULL, 2);
    mbar_init(bar + 8 * L::B_QFREE, 1);
    mbar_init(bar + 8 * L::B_OFULL, 1);
    mbar_init(bar + 8 * L::B_OFREE, F_WARPS);
    mbar_init(bar + 8 * L::B_MLFULL, F_WARPS);
    for (int f = 0; f < F_FACTORS; ++f) mbar_init(bar + 8 * (L::B_FACTORS + f), 2);
    mbar_init(bar + 8 * L::B_DRAIN, 1);
    misc[1] = 0;
    misc[2] = 0;
    mbar_init_fence();
  }
  fence_proxy_async();
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::OFF_MISC), "r"(TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  grid_dependency_wait();
  grid_launch_dependents();
  const int u0 = plan[a.off_tcta + 2 * blockIdx.x], u1 = plan[a.off_tcta + 2 * blockIdx.x + 1];
  const long long limit = pv.wait_limit;
  uint32_t prod_it = 0;       // warp 0: tiles whose copies have been issued
  volatile int *ring = reinterpret_cast<volatile int *>(misc + 2);
  int32_t *counter = pv.status + PASTA_STATUS_TAIL_COUNTER;

  // test hook: a held role goes straight to the tear-down, so that the roles waiting for it run into their limits
  const int role = warp == 0 ? 0 : warp == 1 ? 1 : warp < 4 ? 2 : 3 + ((warp - 4) >> 2);
  if ((pv.debug_hold >> role) & 1) {
  } else if (warp == 0) {
    // ================================================================ producer
    uint32_t it = 0;
    bool ok = true;
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    while (ok && next_unit<true, true>(wk, a, plan, u0, u1, ring, counter, lane, true, abort_flag, limit, ok, x, ll)) {
      const uint8_t *kv_layer = pv.kv_base + (a.layer_begin + ll) * pv.layer_stride;
      // Page ids, metas and scales of a batch of 4 tiles live in registers, a page per lane.  A page's scales sit behind a
      // second trip to memory (page id, then scales), which takes a microsecond or two while the copies saturate it: the
      // ids are asked for two batches ahead and the scales one.  A stage is full when its bytes have landed and its scales
      // have been stored (two arrivals), so that a unit's first copies do not wait for its first scales.
      const uint16_t *scales = reinterpret_cast<const uint16_t *>(kv_layer + pv.scale_off);
      auto ask = [&](int tile, int &page, int &meta) {
        page = 0;
        meta = -1;
        const int at = tile * PASTA_TILE_PAGES + lane;
        if (at < x.n_pages && at < x.tile_end * PASTA_TILE_PAGES) {
          page = plan[a.off_pages + x.page_off + at];
          meta = plan[a.off_pmeta + x.page_off + at];
        }
      };
      auto ask_scales = [&](int &page, int &meta) {
        if (page < 0 || page >= pv.n_pages) { report(pv.status, PASTA_ERR_DEVICE_CHECK); page = 0; meta = -1; }
        return static_cast<int>(scales[static_cast<int64_t>(page) * pv.n_kv_heads + x.g]);
      };
      int page, meta, sc, n1_page, n1_meta, n1_sc = 0, n2_page, n2_meta;       // this batch, the next, the one behind it
      ask(x.tile_begin, page, meta);
      ask(x.tile_begin + 4, n1_page, n1_meta);
      ask(x.tile_begin + 8, n2_page, n2_meta);
      sc = ask_scales(page, meta);
      auto copies = [&](int tile, uint32_t i) {
        const int s = i % F_STAGES;
        const int n_valid = min(PASTA_TILE_PAGES, x.n_pages - tile * PASTA_TILE_PAGES);
        if (i < F_STAGES && n_valid < PASTA_TILE_PAGES) {       // first use of this stage and some slots stay empty
          uint4 *slot = reinterpret_cast<uint4 *>(sm + L::OFF_STAGE + s * F_STAGE_BYTES + n_valid * F_BLOCK);
          for (int j = lane; j < (PASTA_TILE_PAGES - n_valid) * (F_BLOCK / 16); j += 32) slot[j] = make_uint4(0, 0, 0, 0);
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_expect_tx(bar + 8 * (L::B_FULL + s), n_valid * F_BLOCK);
        __syncwarp();
        const int first = ((tile - x.tile_begin) & 3) * PASTA_TILE_PAGES, r = lane - first;
        if (r >= 0 && r < n_valid)
          bulk_g2s_stream(base + L::OFF_STAGE + s * F_STAGE_BYTES + r * F_BLOCK,
                          kv_layer + (static_cast<int64_t>(page) * pv.n_kv_heads + x.g) * F_BLOCK, F_BLOCK,
                          bar + 8 * (L::B_FULL + s), policy);
      };
      auto store_scales = [&](int tile, uint32_t i) {
        const int s = i % F_STAGES, first = ((tile - x.tile_begin) & 3) * PASTA_TILE_PAGES, r = lane - first;
        if (r >= 0 && r < PASTA_TILE_PAGES) {
          meta_s[s * PASTA_TILE_PAGES + r] = meta;
          scale_s[s * PASTA_TILE_PAGES + r] = sc;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + 8 * (L::B_FULL + s));
      };
      int copied = x.tile_begin;                  // tiles of this unit whose copies have been issued
      for (int tile = x.tile_begin; tile < x.tile_end; ++tile, ++it) {
        const bool batch = ((tile - x.tile_begin) & 3) == 0;
        if (batch && tile > x.tile_begin) {
          page = n1_page; meta = n1_meta; sc = n1_sc;
          n1_page = n2_page; n1_meta = n2_meta;
          ask(tile + 8, n2_page, n2_meta);
        }
        if (copied == tile) {
          if (!warp_wait_or_abort(bar + 8 * (L::B_EMPTY + it % F_STAGES), ((it / F_STAGES) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
          copies(tile, it);
          ++copied;
          // the first batch: further tiles whose stages are free already, before the scales are waited for
          for (; tile == x.tile_begin && copied < min(x.tile_end, tile + 4); ++copied) {
            const uint32_t i = it + (copied - tile);
            int free = lane == 0 ? mbar_test_wait(bar + 8 * (L::B_EMPTY + i % F_STAGES), ((i / F_STAGES) & 1) ^ 1) : 0;
            if (!__shfl_sync(0xffffffffu, free, 0)) break;
            copies(copied, i);
          }
        }
        if (batch) n1_sc = ask_scales(n1_page, n1_meta);
        store_scales(tile, it);
        prod_it = it + (copied - tile);
      }
      // (giving up leaves no stage without its second arrival: only the tile whose copies come next is waited for)
    }
  } else if (warp == 1) {
    // ================================================================ MMA issue (one thread)
    if (lane == 0) {
      uint32_t it = 0, uc = 0;
      bool ok = true;
      Walk wk{0, u0, 0};
      UnitInfo x;
      int ll = 0;
      for (; ok && next_unit<false, true>(wk, a, plan, u0, u1, ring, counter, lane, false, abort_flag, limit, ok, x, ll); ++uc) {
        const int nt = x.tile_end - x.tile_begin;
        const uint32_t m_bits = unit_m64<NC>(x.n_threads << g_shift) ? IDESC_M64 : IDESC_M128;
        if (!wait_or_abort(bar + 8 * L::B_QFULL, uc & 1, abort_flag, limit)) { ok = false; break; }
        tc_fence_after();
        for (int k = 0; k <= nt && ok; ++k) {
          if (k < nt) {
            // ---- S[b] = Q . K^T for tile `it` (S[b] was last used by tile it - 2, whose P.V was issued before this)
            const uint32_t s = it % F_STAGES, b = it & 1;
            if (!wait_or_abort(bar + 8 * (L::B_FULL + s), (it / F_STAGES) & 1, abort_flag, limit)) { ok = false; break; }
            tc_fence_after();
            const uint32_t k_addr = base + L::OFF_STAGE + s * F_STAGE_BYTES;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {     // the two terms of Q one after the other, four steps of 32 elements each
              const uint32_t term = ks >> 2, kk = ks & 3;
              mma8_ss(tmem + COL_S + b * T_TILE, smem_desc(base + L::OFF_Q + term * F_Q_TERM + kk * 32, 16, 1024),
                      smem_desc(k_addr + kk * 32, 16, 2048), IDESC_QK8 | m_bits, ks > 0);
            }
            mma_commit(bar + 8 * (L::B_SFULL + b));
            if (k == nt - 1) mma_commit(bar + 8 * L::B_QFREE);       // the Q operand may be replaced once these finish
          }
          if (k > 0) {
            // ---- O_g += P_g . V_g for both halves of tile `it - 1` (when k == nt, `it` already points past it)
            const uint32_t j = it - 1;
            const uint32_t s = j % F_STAGES, b = j & 1;
            if (k == 1 && uc > 0) {   // the unit's first P.V overwrites the accumulators: the previous unit's rows must be read out
              if (!wait_or_abort(bar + 8 * L::B_OFREE, (uc - 1) & 1, abort_flag, limit)) { ok = false; break; }
            }
            const uint32_t v_addr = base + L::OFF_STAGE + s * F_STAGE_BYTES + 1024;
            for (uint32_t g = 0; g < 2 && ok; ++g) {
              if (!wait_or_abort(bar + 8 * (L::B_PFULL + 2 * b + g), (j >> 1) & 1, abort_flag, limit)) { ok = false; break; }
              tc_fence_after();
#pragma unroll
              for (int ks = 0; ks < 6; ++ks) {   // steps of 32 tokens (two pages), the three terms of the weights
                const uint32_t term = ks >> 1, kk = ks & 1;
                mma8_ts(tmem + COL_O + g * 128, tmem + COL_S + b * T_TILE + g * F_HALF + term * 16 + kk * 8,
                        smem_desc(v_addr + (4 * g + 2 * kk) * F_BLOCK, 1024, 2048), IDESC_PV8 | m_bits, (k > 1) || (ks > 0));
              }
            }
            if (!ok) break;
            mma_commit(bar + 8 * (L::B_EMPTY + s));
            if (k == nt) mma_commit(bar + 8 * L::B_OFULL);
          }
          if (k < nt) ++it;
        }
      }
    }
  } else if (warp < 4) {
    // ================================================================ Q operand (64 threads, two to a row)
    const int t64 = tid - 64, half = t64 & 1;
    uint32_t uc = 0;
    bool ok = true;
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    for (; ok && next_unit<false, true>(wk, a, plan, u0, u1, ring, counter, lane, true, abort_flag, limit, ok, x, ll); ++uc) {
      const int rows = x.n_threads << g_shift;
      // the rows an MMA reads: the unit's in every copy, zeros beyond its last
      const int copy_rows = NC == 64 ? (unit_m64<NC>(rows) ? 64 : 128) : NC == 32 ? 64 : unit_m64<NC>(rows) ? 16 : 32;
      constexpr int COPIES = 64 / NC;
#pragma unroll 1
      for (int r0 = 0; r0 < copy_rows; r0 += 32) {
        const int row = r0 + (t64 >> 1);
        uint4 val[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) val[c] = make_uint4(0, 0, 0, 0);
        if (row < rows) {
          const int qn = plan[a.off_tq + x.tq_off + (row >> g_shift)];
          const uint4 *src = reinterpret_cast<const uint4 *>(
              q + ((static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (row & (G - 1))) * 128) + half * 8;
#pragma unroll
          for (int c = 0; c < 8; ++c) val[c] = __ldg(src + c);
        }
        uint32_t m2 = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          m2 = __vmaxu2(__vmaxu2(m2, val[c].x & 0x7fff7fffu),
                        __vmaxu2(__vmaxu2(val[c].y & 0x7fff7fffu, val[c].z & 0x7fff7fffu), val[c].w & 0x7fff7fffu));
        int amax = static_cast<int>(max(m2 >> 16, m2 & 0xffffu));
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        const int up = max(-126, min(126, 7 - ((amax >> 7) - 127)));
        const float f = pow2f(up);
#pragma unroll
        for (int c = 0; c < 8; ++c) {             // val becomes the half row's 64 + 64 bytes
          uint32_t h0, l0, h1, l1;
          split_query4(bf16_lo(val[c].x) * f, bf16_hi(val[c].x) * f, bf16_lo(val[c].y) * f, bf16_hi(val[c].y) * f, h0, l0);
          split_query4(bf16_lo(val[c].z) * f, bf16_hi(val[c].z) * f, bf16_lo(val[c].w) * f, bf16_hi(val[c].w) * f, h1, l1);
          val[c] = make_uint4(h0, h1, l0, l1);
        }
        if (r0 == 0 && uc > 0 && !warp_wait_or_abort(bar + 8 * L::B_QFREE, (uc - 1) & 1, abort_flag, limit)) { ok = false; break; }
        // A row's factor is read by the softmax threads of this unit.  The place of unit uc is written again for unit uc + 4,
        // after Q.K^T of unit uc + 3 and hence P.V of unit uc + 2 has been issued: the softmax of unit uc is long over.
        // A row that is not finite says so by its factor: the codes it became are.
        if (half == 0 && row < rows)
          factor_s[(uc % F_FACTORS) * 128 + row] = amax >= 0x7f80 ? NAN : fmaxf(a.scale_log2 * pow2f(-up), 1e-30f);
        if (row < copy_rows)
#pragma unroll
          for (int copy = 0; copy < COPIES; ++copy) {
            const int at_row = copy * copy_rows + row, r8 = at_row & 7;
            uint8_t *dst = sm + L::OFF_Q + at_row * 128;
#pragma unroll
            for (int c = 0; c < 4; ++c) {         // 16 codes of a term: two of val's entries
              const int at = ((half * 4 + c) ^ r8) << 4;
              *reinterpret_cast<uint4 *>(dst + at) = make_uint4(val[2 * c].x, val[2 * c].y, val[2 * c + 1].x, val[2 * c + 1].y);
              *reinterpret_cast<uint4 *>(dst + F_Q_TERM + at) = make_uint4(val[2 * c].z, val[2 * c].w, val[2 * c + 1].z, val[2 * c + 1].w);
            }
          }
      }
      if (!ok) break;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar + 8 * (L::B_FACTORS + uc % F_FACTORS));
        mbar_arrive(bar + 8 * L::B_QFULL);
      }
    }
  } else {
    // ================================================================ softmax + epilogue (2 groups of 128 threads)
    const int grp = (warp - 4) >> 2;              // this group's half of every tile: pages 4 grp .. 4 grp + 3
    const int wq = warp & 3;                      // the quarter of TMEM this warp reaches: lanes 32 wq .. 32 wq + 31
    const uint32_t lane_addr = static_cast<uint32_t>(wq * 32) << 16;
    constexpr int PAGES = NC / 16;                // of this thread's columns
    const int page0 = NC == 16 ? wq : NC == 32 ? 2 * (wq >> 1) : 0;       // the first of them within the group's four
    const bool keeps = NC == 64 || (NC == 32 ? wq < 2 : wq == 0);         // the copy that ends up with the sum
    const float cap = pv.softcap_log2;
    uint32_t it = 0, uc = 0;
    bool ok = true;
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    for (; ok && next_unit<false, true>(wk, a, plan, u0, u1, ring, counter, lane, true, abort_flag, limit, ok, x, ll); ++uc) {
      const int nt = x.tile_end - x.tile_begin;
      const int rows = x.n_threads << g_shift;
      const bool m64 = unit_m64<NC>(rows);
      const int row = NC == 16 ? lane : NC == 32 ? (wq & 1) * 32 + lane : m64 ? wq * 16 + lane : wq * 32 + lane;
      const bool active = row < rows && !(m64 && lane >= 16);
      const bool warp_active = NC < 64 || (m64 ? wq * 16 : wq * 32) < rows;
      const int vis_at = a.off_vis + x.vis_off + (active ? row >> g_shift : 0) * x.n_streams;
      const int vis0 = plan[vis_at];
      const bool fin = x.final_rows != 0;         // for the epilogue: looked up here, where the wait for it is hidden
      const int qn = active && keeps && fin ? plan[a.off_tq + x.tq_off + (row >> g_shift)] : 0;
      if (!warp_wait_or_abort(bar + 8 * (L::B_FACTORS + uc % F_FACTORS), (uc / F_FACTORS) & 1, abort_flag, limit)) { ok = false; break; }
      const float factor = active ? factor_s[(uc % F_FACTORS) * 128 + row] : 1.f;
      float ref = -INFINITY, l = 0.f;
      for (int k = 0; k < nt; ++k, ++it) {
        const uint32_t s = it % F_STAGES, b = it & 1;
        const uint32_t s_addr = tmem + lane_addr + COL_S + b * T_TILE + grp * F_HALF;
        // (the scores' barrier stands behind the stage's: the MMA thread has seen that one complete)
        if (!warp_wait_or_abort(bar + 8 * (L::B_SFULL + b), (it >> 1) & 1, abort_flag, limit)) { ok = false; break; }
        tc_fence_after();
        if (warp_active) {
          float sc[NC], c_pg[PAGES], mt = -INFINITY;
          uint32_t *sr = reinterpret_cast<uint32_t *>(sc);
          if constexpr (NC == 16) {
            tmem_ld16_issue(s_addr + page0 * 16, sr);
          } else if constexpr (NC == 32) {
            tmem_ld32_issue(s_addr + page0 * 16, sr);
          } else {
            tmem_ld32_issue(s_addr, sr);
            tmem_ld32_issue(s_addr + 32, sr + 32);
          }
          int meta[PAGES], sc2[PAGES], thr[PAGES];
          const int at = s * PASTA_TILE_PAGES + grp * 4 + page0;
          if constexpr (PAGES == 4) {
            *reinterpret_cast<int4 *>(meta) = *reinterpret_cast<const int4 *>(meta_s + at);
            *reinterpret_cast<int4 *>(sc2) = *reinterpret_cast<const int4 *>(scale_s + at);
          } else if constexpr (PAGES == 2) {
            *reinterpret_cast<int2 *>(meta) = *reinterpret_cast<const int2 *>(meta_s + at);
            *reinterpret_cast<int2 *>(sc2) = *reinterpret_cast<const int2 *>(scale_s + at);
          } else {
            meta[0] = meta_s[at];
            sc2[0] = scale_s[at];
          }
          // pages that every thread of the request sees in full need no thresholds
          bool full = true;
#pragma unroll
          for (int pg = 0; pg < PAGES; ++pg) full = full && meta[pg] >= 0 && (meta[pg] & PASTA_PMETA_ALL_VISIBLE);
          if (!full) {
            full = true;
#pragma unroll
            for (int pg = 0; pg < PAGES; ++pg) {
              thr[pg] = PASTA_PAGE;
              if (!(meta[pg] >= 0 && (meta[pg] & PASTA_PMETA_ALL_VISIBLE))) {
                int t = 0;
                if (active && meta[pg] >= 0) {
                  const int sl = PASTA_PMETA_STREAM(meta[pg]);
                  const int vis = sl == 0 ? vis0 : plan[vis_at + sl];
                  t = min(max(vis - PASTA_PMETA_PAGE(meta[pg]) * PASTA_PAGE, 0), PASTA_PAGE);
                }
                thr[pg] = t;
                full = full && t == PASTA_PAGE;
              }
            }
          }
          if constexpr (NC == 16) {
            asm volatile("tcgen05.wait::ld.sync.aligned;" : PASTA_RW16(sr) :: "memory");
          } else {
            tmem_ld_wait32(sr);
            if constexpr (NC == 64) tmem_ld_order32(sr + 32);
          }
          // a page brings a factor of its own (its K's scale) and an addend (its V's exponent, which the weights carry)
#pragma unroll
          for (int pg = 0; pg < PAGES; ++pg) c_pg[pg] = fmaxf(code_factor(factor, static_cast<int8_t>(sc2[pg] & 0xff)), 1e-37f);   // never 0: it meets -inf
          if (kCap) {
#pragma unroll
            for (int j = 0; j < NC; ++j) sc[j] *= capped_factor(c_pg[j >> 4], a.cap_inv);
            softcap_columns<NC>(sc, cap, active);
#pragma unroll
            for (int pg = 0; pg < PAGES; ++pg) c_pg[pg] = 1.f;    // capped scores are in log2 units from here on
          }
          if (!full) {
#pragma unroll
            for (int j = 0; j < NC; ++j)
              if ((j & 15) >= thr[j >> 4]) sc[j] = -INFINITY;
          }
#pragma unroll
          for (int pg = 0; pg < PAGES; ++pg) {
            float m0 = fmaxf(sc[16 * pg], sc[16 * pg + 1]), m1 = fmaxf(sc[16 * pg + 2], sc[16 * pg + 3]);
#pragma unroll
            for (int j = 4; j < 16; j += 4) {
              m0 = fmaxf(fmaxf(m0, sc[16 * pg + j]), sc[16 * pg + j + 1]);
              m1 = fmaxf(fmaxf(m1, sc[16 * pg + j + 2]), sc[16 * pg + j + 3]);
            }
            mt = fmaxf(mt, fmaf(fmaxf(m0, m1), c_pg[pg], static_cast<float>(static_cast<int8_t>(sc2[pg] >> 8))));
          }
          // Far from 0 a rounded maximum and an unrounded score may differ by more than the terms have room for: such a row's scores
          // are rounded as its maximum was, and taken relative to it, before the reference is subtracted.
          const bool far = !kCap && fabsf(mt) > FAR_SCORE && fabsf(mt) < INFINITY;      // (a cap keeps scores below 2^21)
          if (!kCap && __any_sync(0xffffffffu, active && far)) {
#pragma unroll
            for (int pg = 0; pg < PAGES; ++pg) {
#pragma unroll
              for (int j = 16 * pg; j < 16 * pg + 16; ++j)
                sc[j] = far ? fmaf(sc[j], c_pg[pg], static_cast<float>(static_cast<int8_t>(sc2[pg] >> 8))) - mt : sc[j];
              c_pg[pg] = far ? 1.f : c_pg[pg];
            }
          }
          const bool need = mt > ref + P_SLACK;       // also true for the first visible tile (ref = -inf)
          const bool rescale = active && need && l > 0.f;
          const float set = kCap || fabsf(mt) < 32 * FAR_SCORE ? mt - P_TOP : mt;      // exact: beyond, fp32 steps are 4 and more
          if (__any_sync(0xffffffffu, rescale)) {
            // O_g and l are relative to ref: move them to the new reference.  The accumulator is quiet once the P.V of the
            // previous tile has finished, which is what releases that tile's stage.
            if (!warp_wait_or_abort(bar + 8 * (L::B_EMPTY + (it - 1) % F_STAGES), ((it - 1) / F_STAGES) & 1, abort_flag, limit)) { ok = false; break; }
            tc_fence_after();
            const float f = rescale ? fast_exp2(ref - set) : 1.f;
#pragma unroll 1
            for (int h = 0; h < 128; h += 16) {
              uint32_t ov[16];
              const uint32_t at = tmem + lane_addr + COL_O + grp * 128 + h;
              tmem_ld16(at, ov);
#pragma unroll
              for (int j = 0; j < 16; ++j) ov[j] = __float_as_uint(__uint_as_float(ov[j]) * f);
#pragma unroll
              for (int j = 0; j < 16; j += 4) tmem_st4(at + j, ov[j], ov[j + 1], ov[j + 2], ov[j + 3]);
            }
            tmem_st_wait();
            l *= f;
          }
          if (need) ref = set;
          const float rf = ref == -INFINITY ? 0.f : ref == INFINITY ? NAN : ref;      // a score beyond fp32 spoils its row
          // weights as three e5m2 terms, four to a column, where scores were that are in registers by now; l sums them unrounded
          // and without V's scale, page by page
#pragma unroll
          for (int pg = 0; pg < PAGES; ++pg) {
            const int ev = static_cast<int8_t>(sc2[pg] >> 8);
            const float add = (far ? mt : static_cast<float>(ev)) - rf;
            float ls[2] = {0.f, 0.f};
            uint32_t t[4][3];
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              float x0, x1, x2, x3;
              fma2(x0, x1, sc[16 * pg + j], sc[16 * pg + j + 1], c_pg[pg], add);
              fma2(x2, x3, sc[16 * pg + j + 2], sc[16 * pg + j + 3], c_pg[pg], add);
              const float p0 = fast_exp2(x0), p1 = fast_exp2(x1), p2 = fast_exp2(x2), p3 = fast_exp2(x3);
              add2(ls[0], ls[1], p0, p1);
              add2(ls[0], ls[1], p2, p3);
              split4(p0, p1, p2, p3, t[j >> 2]);
            }
            l = fmaf(ls[0] + ls[1], pow2f(-ev), l);
#pragma unroll
            for (int k = 0; k < 3; ++k) tmem_st4(s_addr + 16 * k + 4 * (page0 + pg), t[0][k], t[1][k], t[2][k], t[3][k]);
          }
#pragma unroll
          for (int pg = PAGES; pg < 4; ++pg)      // zeros for the columns that other copies answer for
#pragma unroll
            for (int k = 0; k < 3; ++k) tmem_st4(s_addr + 16 * k + 4 * ((page0 + pg) & 3), 0, 0, 0, 0);
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + 8 * (L::B_PFULL + 2 * b + grp));
      }
      if (!ok) break;

      // ---- epilogue: a row's accumulators, one per group and copy, leave TMEM brought to one reference and added up, 64
      // columns per group.  The references and sums go through shared memory; so do the accumulators of copies 1 .. (two slots
      // of 8 KB per group, a column per 128 bytes).
      ml_s[((uc & 1) * F_WARPS + warp - 4) * 32 + lane] = make_float2(ref, factor == factor ? l : NAN);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + 8 * L::B_MLFULL);
      if (!warp_wait_or_abort(bar + 8 * L::B_MLFULL, uc & 1, abort_flag, limit) || !warp_wait_or_abort(bar + 8 * L::B_OFULL, uc & 1, abort_flag, limit)) { ok = false; break; }
      tc_fence_after();
      if (warp_active) {
        constexpr int COPIES = 64 / NC;
        float m_all = -INFINITY, l_all = 0.f, l_plain = 0.f;
        float2 part[2 * COPIES];
#pragma unroll
        for (int i = 0; i < 2 * COPIES; ++i) {
          const int w = (i & 1) * 4 + (NC == 64 ? wq : NC == 32 ? (wq & 1) + (i >> 1) * 2 : i >> 1);
          part[i] = ml_s[((uc & 1) * F_WARPS + w) * 32 + lane];
          if (part[i].y > 0.f) m_all = fmaxf(m_all, part[i].x);
          l_plain += part[i].y;
        }
#pragma unroll
        for (int i = 0; i < 2 * COPIES; ++i)
          if (part[i].y > 0.f) l_all = fmaf(part[i].y, fast_exp2(part[i].x - m_all), l_all);
        const bool spoilt = l_plain != l_plain;
        if (spoilt) { m_all = not_a_row().x; l_all = not_a_row().y; }
        // what this lane's two accumulators (one per group) are multiplied by; a factor of 0 means that the accumulator of
        // this row is not looked at
        const int mine = NC == 64 ? 0 : NC == 32 ? wq >> 1 : wq;
        const bool any = l_all > 0.f;             // a row that saw nothing: zeros in the output, nothing in the partial rows
        const float inv = fin && any ? 1.f / l_all : 1.f;
        float f0 = 0.f, f1 = 0.f;
#pragma unroll
        for (int i = 0; i < COPIES; ++i)
          if (i == mine) {
            f0 = part[2 * i].y > 0.f ? fast_exp2(part[2 * i].x - m_all) * inv : 0.f;
            f1 = part[2 * i + 1].y > 0.f ? fast_exp2(part[2 * i + 1].x - m_all) * inv : 0.f;
          }
        if (spoilt) f0 = f1 = NAN;
        const uint32_t o_addr = tmem + lane_addr + COL_O + grp * 64;
        float *slots = reinterpret_cast<float *>(sm + L::OFF_SUM + grp * F_SUM_BYTES) + lane;
        auto folded = [&](int h, float *v) {      // 16 of the group's columns, both accumulators
          uint32_t r0[16], r1[16];
          tmem_ld16_issue(o_addr + h, r0);
          tmem_ld16_issue(o_addr + 128 + h, r1);
          tmem_ld_wait16x2(r0, r1);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            v[j] = (f0 != 0.f ? f0 * __uint_as_float(r0[j]) : 0.f) + (f1 != 0.f ? f1 * __uint_as_float(r1[j]) : 0.f);
        };
        auto meet = [&](uint32_t n) {             // the group's four warps; n: how many times before this
          __syncwarp();
          if (lane == 0) mbar_arrive(bar + 8 * (L::B_SUM + grp));
          return warp_wait_or_abort(bar + 8 * (L::B_SUM + grp), n & 1, abort_flag, limit);
        };
        if (NC < 64) {
          if (wq >= 2) {
#pragma unroll 1
            for (int h = 0; h < 64; h += 16) {
              float v[16];
              folded(h, v);
#pragma unroll
              for (int j = 0; j < 16; ++j) slots[(wq - 2) * 2048 + (h + j) * 32] = v[j];
            }
          }
          if (!meet(NC == 16 ? 2 * uc : uc)) { ok = false; break; }
        }
        if (NC == 16) {
          if (wq == 1) {
#pragma unroll 1
            for (int h = 0; h < 64; h += 16) {
              float v[16];
              folded(h, v);
#pragma unroll
              for (int j = 0; j < 16; ++j) slots[2048 + (h + j) * 32] += v[j];
            }
          }
          if (!meet(2 * uc + 1)) { ok = false; break; }
        }
        if (keeps) {
          const int64_t at_row = fin ? (static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (row & (G - 1))
                                     : static_cast<int64_t>(ll) * pv.rows_per_layer + x.row_base + row;
#pragma unroll 1
          for (int h = 0; h < 64; h += 16) {
            float v[16];
            folded(h, v);
            if (NC == 32) {
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] += slots[wq * 2048 + (h + j) * 32];
            }
            if (NC == 16) {
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] = (v[j] + slots[(h + j) * 32]) + slots[2048 + (h + j) * 32];
            }
            if (!active) continue;
            if (fin && a.out_bf16) {
              uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at_row * 128 + grp * 64 + h);
#pragma unroll
              for (int j = 0; j < 2; ++j)
                dst[j] = make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]),
                                    pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
            } else if (fin || any) {
              float4 *dst = reinterpret_cast<float4 *>((fin ? static_cast<float *>(a.out) : pv.part_o) + at_row * 128 + grp * 64 + h);
#pragma unroll
              for (int j = 0; j < 4; ++j) dst[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
          }
          if (grp == 0 && active) {
            if (!fin) pv.part_ml[at_row] = make_float2(m_all, l_all);
            else if (a.lse) a.lse[at_row] = (m_all + log2f(l_all)) * 0.6931471805599453f;
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + 8 * L::B_OFREE);
    }
  }

  // ---- tear-down
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // see attn_tensor.cu: what is still in flight for this CTA (bulk copies, MMAs) ends on its own and is waited for
    if (warp == 0 && lane == 0) {
      for (uint32_t j = (prod_it > F_STAGES ? prod_it - F_STAGES : 0); j < prod_it; ++j)
        mbar_wait_bounded(bar + 8 * (L::B_FULL + j % F_STAGES), (j / F_STAGES) & 1);
    }
    if (warp == 1 && lane == 0) {
      mma_commit(bar + 8 * L::B_DRAIN);
      mbar_wait_bounded(bar + 8 * L::B_DRAIN, 0);
    }
    if (tid == 0) report(pv.status, PASTA_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
  }
  if (warp == 2) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
  }
}

}  // namespace

template <int NC>
static cudaError_t launch_t(const PoolView &pv, const PlanHeader &h, int32_t layer_begin, int32_t layer_count,
                            const void *q, float scale_log2, void *out, float *lse, bool out_bf16, cudaStream_t st) {
  static uint64_t prepared[2] = {0, 0};
  const bool cap = pv.softcap_log2 > 0.f;
  const auto kernel = cap ? attn_kv8_tensor_kernel<NC, true> : attn_kv8_tensor_kernel<NC, false>;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void *>(kernel), F<NC>::SMEM_BYTES, &prepared[cap]);
  if (e != cudaSuccess) return e;
  const int grid = h.w[PH_T_GRID];
  if (grid == 0 || layer_count == 0) return cudaSuccess;
  TensorArgs a;
  a.off_tunit = h.w[PH_OFF_TUNIT]; a.off_treq = h.w[PH_OFF_TREQ]; a.off_tcta = h.w[PH_OFF_TCTA];
  a.off_pages = h.w[PH_OFF_PAGES]; a.off_pmeta = h.w[PH_OFF_PMETA]; a.off_vis = h.w[PH_OFF_VIS];
  a.off_tq = h.w[PH_OFF_TQ];
  a.off_dunit = h.w[PH_OFF_DUNIT]; a.n_dunits = h.w[PH_N_DUNITS];
  a.n_queries = h.w[PH_N_QUERIES]; a.layer_begin = layer_begin; a.layer_count = layer_count;
  a.scale_log2 = scale_log2;
  a.cap_inv = cap ? 1.f / pv.softcap_log2 : 0.f;
  a.out = out; a.lse = lse; a.out_bf16 = out_bf16 ? 1 : 0;
  return launch_overlapped(kernel, dim3(grid), dim3(F_THREADS), F<NC>::SMEM_BYTES, st, pv, a, static_cast<const __nv_bfloat16 *>(q));
}

cudaError_t launch_attn_kv8_tensor(const PoolView &pv, const PlanHeader &h, int32_t layer_begin, int32_t layer_count,
                                   const void *q, float scale_log2, void *out, float *lse, bool out_bf16, cudaStream_t st) {
  if (pv.head_dim != 128) return cudaErrorInvalidValue;
  const int rows = h.w[PH_T_MAX_ROWS];
  return rows <= 32 ? launch_t<16>(pv, h, layer_begin, layer_count, q, scale_log2, out, lse, out_bf16, st)
       : rows <= 64 ? launch_t<32>(pv, h, layer_begin, layer_count, q, scale_log2, out, lse, out_bf16, st)
                    : launch_t<64>(pv, h, layer_begin, layer_count, q, scale_log2, out, lse, out_bf16, st);
}

}  // namespace pasta
