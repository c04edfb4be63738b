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
// tokens, and the weights of those tokens are N further columns: [V_0; V_1] [P_0 | P_1], K = 64.  The two diagonal blocks are
// what is wanted and are added up at a unit's end; the other two cost nothing that matters at these N.
//
// The reference of a row is shared by the tokens of a tile, that is by the four warps of a softmax group, so raising it takes
// an agreement: every tile the group votes whether some score lies more than 2^R_SLACK above its row's reference (also: whether a
// row sees its first token), and only then are the rows' maxima worked out, and O and l brought to the new reference.
//
// Warp roles (640 threads): warp 0 producer (bulk copies), warp 1 MMA issue (one thread, Q.K^T one tile ahead of P.V), warps 2-3
// build the Q operand, warps 4-7 turn K's codes into the A operand, warps 8-11 V's, warps 12-15 and 16-19 are two softmax
// groups, which take the rows in turn, eight at a time.  Every wait is bounded; on expiry the CTA reports PASTA_ERR_TIMEOUT, drains
// and leaves.
#include "tensor_common.cuh"

namespace pasta {

namespace {

constexpr int U_THREADS = 640;
constexpr int U_RING = 32;                       // unit records and tiles' page metas kept published: more than the pipeline is deep
constexpr int U_INIT = 4;                        // units whose rows' first references are kept
constexpr float R_SLACK = 10.f;                  // weights are at most 2^10 (bf16 and fp32 keep their precision at any size)
constexpr float R_UNSET = 3e38f;                 // minus the reference of a row that has seen nothing

// Sizes of one build: head_dim D, at most NMAX stacked rows.
template <int D, int NMAX>
struct U {
  static constexpr int CHUNKS = NMAX / 16;                        // groups of 8 rows per softmax group
  static constexpr int OW = D == 128 ? 1 : 2;                     // blocks of N columns of an accumulator
  static constexpr int KSTEPS = D / 16, VSTEPS = D == 128 ? 8 : 4;
  static constexpr int KW = D / 2, VW = VSTEPS * 8;               // TMEM columns of a K and a V operand
  // how many of each fit 512 columns
  static constexpr int SB = D == 64 && NMAX > 96 ? 1 : 2, OB = NMAX > 64 ? 1 : 2;
  static constexpr int KB = D == 128 && NMAX > 96 ? 1 : 2, VB = D == 128 && NMAX > 64 ? 1 : 2;
  static constexpr int QB = NMAX > 64 ? 1 : 2;
  static constexpr uint32_t COL_S = 0, COL_O = COL_S + SB * NMAX, COL_K = COL_O + OB * OW * NMAX, COL_V = COL_K + KB * KW;
  static_assert(COL_V + VB * VW <= TMEM_COLS, "tensor memory budget");
  static constexpr int BLOCK = kv4_block_bytes(D), STAGE_BYTES = PASTA_TILE_PAGES * BLOCK;
  static constexpr int ATOMS = (OW * NMAX + 63) / 64;             // 64-column atoms of a weight row
  static constexpr int P_BYTES = (D == 128 ? 16 : 8) * ATOMS * 1024;
  static constexpr int Q_BYTES = NMAX * D * 2;
  static constexpr int SUM_BYTES = D == 64 ? NMAX * 64 * 4 : 0;   // where the halves of accumulators are added up
  static constexpr int STAGES = D == 64 ? 10 : NMAX > 64 ? 6 : 7;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_P = OFF_Q + QB * Q_BYTES;
  static constexpr int OFF_STAGE = OFF_P + 2 * P_BYTES;
  static constexpr int OFF_SUM = OFF_STAGE + STAGES * STAGE_BYTES;
  static constexpr int OFF_BAR = OFF_SUM + SUM_BYTES;
  // barriers (8 bytes each)
  static constexpr int B_FULL = 0, B_EMPTY = B_FULL + STAGES, B_KFULL = B_EMPTY + STAGES, B_KFREE = B_KFULL + KB,
                       B_VFULL = B_KFREE + KB, B_VFREE = B_VFULL + VB, B_SFULL = B_VFREE + VB, B_SFREE = B_SFULL + SB,
                       B_PFULL = B_SFREE + SB, B_PFREE = B_PFULL + 2, B_QFULL = B_PFREE + 2, B_QFREE = B_QFULL + QB,
                       B_OFULL = B_QFREE + QB, B_OFREE = B_OFULL + OB,
                       B_SYNC = B_OFREE + OB,                       // [group] where a softmax group meets
                       B_DRAIN = B_SYNC + 2,                        // only used when a role gave up
                       B_COUNT = B_DRAIN + 1;
  static constexpr int OFF_META = OFF_BAR + 8 * ((B_COUNT + 1) & ~1);        // [U_RING] 8 page metas
  static constexpr int OFF_MISC = OFF_META + U_RING * 32;                  // tmem base, abort flag, shared units taken, their records
  static constexpr int OFF_INIT = OFF_MISC + 16 + 64 * U_RING;             // [U_INIT][NMAX] rows' first references (negated)
  static constexpr int OFF_REF = OFF_INIT + U_INIT * NMAX * 4;             // [NMAX] references (negated)
  static constexpr int OFF_FACT = OFF_REF + NMAX * 4;                      // [NMAX] what a raised reference multiplies O and l by; 1 / l
  static constexpr int OFF_WARP = OFF_FACT + NMAX * 4;                     // [4][NMAX] a warp's maxima, or sums
  static constexpr int OFF_VOTE = OFF_WARP + 4 * NMAX * 4;                 // [group][4] votes of the latest tiles
  static constexpr int SMEM_BYTES = OFF_VOTE + 32 + 1024;                  // slack to align the base to 1024
  static_assert(SMEM_BYTES <= 232448, "shared memory budget");
  static_assert(OFF_META % 16 == 0 && OFF_MISC % 16 == 0 && OFF_REF % 16 == 0, "read as vectors");
  static_assert(STAGES + KB + SB + 4 <= U_RING, "records are overwritten only after their last reader");
};

constexpr uint32_t IDESC4 = (1u << 4) | (1u << 7) | (1u << 10) | IDESC_M128;      // D fp32, A and B bf16, M = 128
constexpr uint32_t IDESC4_PV = IDESC4 | (1u << 16);                                // B (= P^T) MN-major

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

template <int D, int NMAX, bool kCap>
__global__ void __launch_bounds__(U_THREADS, 1)
attn_kv4_kernel(PoolView pv, TensorArgs a, const __nv_bfloat16 *__restrict__ q) {
  using L = U<D, NMAX>;
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
  volatile int *abort_flag = reinterpret_cast<volatile int *>(misc + 1);
  float *init_s = reinterpret_cast<float *>(sm + L::OFF_INIT);
  const int32_t *plan = pv.plan;

  if (tid == 0) {
    for (int s = 0; s < L::STAGES; ++s) { mbar_init(bar + 8 * (L::B_FULL + s), 1); mbar_init(bar + 8 * (L::B_EMPTY + s), 8); }
    for (int b = 0; b < L::KB; ++b) { mbar_init(bar + 8 * (L::B_KFULL + b), 4); mbar_init(bar + 8 * (L::B_KFREE + b), 1); }
    for (int b = 0; b < L::VB; ++b) { mbar_init(bar + 8 * (L::B_VFULL + b), 4); mbar_init(bar + 8 * (L::B_VFREE + b), 1); }
    for (int b = 0; b < L::SB; ++b) { mbar_init(bar + 8 * (L::B_SFULL + b), 1); mbar_init(bar + 8 * (L::B_SFREE + b), 8); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar + 8 * (L::B_PFULL + b), 8); mbar_init(bar + 8 * (L::B_PFREE + b), 1); }
    for (int b = 0; b < L::QB; ++b) { mbar_init(bar + 8 * (L::B_QFULL + b), 2); mbar_init(bar + 8 * (L::B_QFREE + b), 1); }
    for (int b = 0; b < L::OB; ++b) { mbar_init(bar + 8 * (L::B_OFULL + b), 1); mbar_init(bar + 8 * (L::B_OFREE + b), 8); }
    for (int b = 0; b < 2; ++b) mbar_init(bar + 8 * (L::B_SYNC + b), 4);
    mbar_init(bar + 8 * L::B_DRAIN, 1);
    misc[1] = 0;
    misc[2] = 0;
    for (int i = 0; i < 8; ++i) reinterpret_cast<int *>(sm + L::OFF_VOTE)[i] = 0;
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
  auto next = [&](Walk &w, bool whole_warp, bool &ok, UnitInfo &x, int &ll) {
    return next_unit<false, true, U_RING>(w, a, plan, u0, u1, ring, counter, lane, whole_warp, abort_flag, limit, ok, x, ll);
  };
  auto rows16 = [&](const UnitInfo &x) { return ((x.n_threads << g_shift) + 15) & ~15; };

  // test hook: a held role goes straight to the tear-down, so that the roles waiting for it run into their limits
  const int role = warp == 0 ? 0 : warp < 12 ? (warp == 1 || warp >= 4 ? 1 : 2) : 3 + ((warp - 12) >> 2);
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
    while (ok && next_unit<true, true, U_RING>(wk, a, plan, u0, u1, ring, counter, lane, true, abort_flag, limit, ok, x, ll)) {
      const uint8_t *kv_layer = pv.kv_base + (a.layer_begin + ll) * pv.layer_stride;
      // page ids and metas of a batch of 4 tiles live in registers, a page per lane; the next batch's are asked for ahead
      auto ask = [&](int tile, int &page, int &meta) {
        page = 0;
        meta = -1;
        const int at = tile * PASTA_TILE_PAGES + lane;
        if (at < x.n_pages && at < x.tile_end * PASTA_TILE_PAGES) {
          page = plan[a.off_pages + x.page_off + at];
          meta = plan[a.off_pmeta + x.page_off + at];
        }
      };
      int page, meta, next_page, next_meta;
      ask(x.tile_begin, page, meta);
      ask(x.tile_begin + 4, next_page, next_meta);
      for (int tile = x.tile_begin; tile < x.tile_end; ++tile, ++it) {
        const int first = ((tile - x.tile_begin) & 3) * PASTA_TILE_PAGES, r = lane - first;
        if (first == 0 && tile > x.tile_begin) {
          page = next_page;
          meta = next_meta;
          ask(tile + 4, next_page, next_meta);
        }
        const int s = it % L::STAGES;
        if (!warp_wait_or_abort(bar + 8 * (L::B_EMPTY + s), ((it / L::STAGES) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
        const int n_valid = min(PASTA_TILE_PAGES, x.n_pages - tile * PASTA_TILE_PAGES);
        if (page < 0 || page >= pv.n_pages) { report(pv.status, PASTA_ERR_DEVICE_CHECK); page = 0; meta = -1; }
        if (r >= 0 && r < PASTA_TILE_PAGES) meta_s[(it % U_RING) * PASTA_TILE_PAGES + r] = meta;
        uint8_t *stage = sm + L::OFF_STAGE + s * L::STAGE_BYTES;
        if (it < L::STAGES && n_valid < PASTA_TILE_PAGES) {       // first use of this stage and some slots stay empty
          uint4 *slot = reinterpret_cast<uint4 *>(stage + n_valid * L::BLOCK);
          for (int i = lane; i < (PASTA_TILE_PAGES - n_valid) * (L::BLOCK / 16); i += 32) slot[i] = make_uint4(0, 0, 0, 0);
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_expect_tx(bar + 8 * (L::B_FULL + s), n_valid * L::BLOCK);
        __syncwarp();
        if (r >= 0 && r < n_valid)
          bulk_g2s_stream(base + L::OFF_STAGE + s * L::STAGE_BYTES + r * L::BLOCK,
                          kv_layer + (static_cast<int64_t>(page) * pv.n_kv_heads + x.g) * L::BLOCK, L::BLOCK,
                          bar + 8 * (L::B_FULL + s), policy);
      }
    }
    prod_it = it;
  } else if (warp == 1) {
    // ================================================================ MMA issue (one thread)
    if (lane == 0) {
      uint32_t it = 0, uc = 0;
      bool ok = true;
      Walk wk{0, u0, 0};
      UnitInfo x;
      int ll = 0;
      for (; ok && next(wk, false, ok, x, ll); ++uc) {
        const int nt = x.tile_end - x.tile_begin;
        const uint32_t n = rows16(x), qb = uc % L::QB, ob = uc % L::OB;
        const uint32_t i_qk = IDESC4 | ((n >> 3) << 17), i_pv = IDESC4_PV | (((L::OW * n) >> 3) << 17);
        if (!wait_or_abort(bar + 8 * (L::B_QFULL + qb), (uc / L::QB) & 1, abort_flag, limit)) { ok = false; break; }
        for (int k = 0; k <= nt && ok; ++k) {
          if (k < nt) {
            // ---- S^T = K . Q^T for tile `it`
            const uint32_t kb = it % L::KB, sb = it % L::SB;
            if (!wait_or_abort(bar + 8 * (L::B_SFREE + sb), ((it / L::SB) & 1) ^ 1, abort_flag, limit) ||
                !wait_or_abort(bar + 8 * (L::B_KFULL + kb), (it / L::KB) & 1, abort_flag, limit)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int ks = 0; ks < L::KSTEPS; ++ks)
              mma_ts(tmem + L::COL_S + sb * NMAX, tmem + L::COL_K + kb * L::KW + ks * 8,
                     smem_desc(base + L::OFF_Q + qb * L::Q_BYTES + (ks >> 2) * (NMAX * 128) + (ks & 3) * 32, 16, 1024), i_qk, ks > 0);
            mma_commit(bar + 8 * (L::B_SFULL + sb));
            mma_commit(bar + 8 * (L::B_KFREE + kb));
            if (k == nt - 1) mma_commit(bar + 8 * (L::B_QFREE + qb));   // the Q operand may be replaced once these finish
          }
          if (k > 0) {
            // ---- O^T += V^T . P^T for tile `it - 1` (when k == nt, `it` already points past it)
            const uint32_t j = it - 1, vb = j % L::VB, pb = j & 1;
            if (k == 1 && !wait_or_abort(bar + 8 * (L::B_OFREE + ob), ((uc / L::OB) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
            if (!wait_or_abort(bar + 8 * (L::B_VFULL + vb), (j / L::VB) & 1, abort_flag, limit) ||
                !wait_or_abort(bar + 8 * (L::B_PFULL + pb), (j >> 1) & 1, abort_flag, limit)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int ks = 0; ks < L::VSTEPS; ++ks)
              mma_ts(tmem + L::COL_O + ob * L::OW * NMAX, tmem + L::COL_V + vb * L::VW + ks * 8,
                     smem_desc(base + L::OFF_P + pb * L::P_BYTES + ks * 2 * L::ATOMS * 1024, 1024, L::ATOMS * 1024), i_pv, (k > 1) || (ks > 0));
            mma_commit(bar + 8 * (L::B_VFREE + vb));
            mma_commit(bar + 8 * (L::B_PFREE + pb));
            if (k == nt) mma_commit(bar + 8 * (L::B_OFULL + ob));
          }
          if (k < nt) ++it;
        }
      }
    }
  } else if (warp < 4) {
    // ================================================================ stacked Q operand (64 threads, four to a row)
    constexpr int PER = D / 32;                  // 16-byte chunks of a thread
    const int t64 = tid - 64, part = t64 & 3;
    uint32_t uc = 0;
    bool ok = true;
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    for (; ok && next(wk, true, ok, x, ll); ++uc) {
      const int rows = x.n_threads << g_shift, n = rows16(x), qb = uc % L::QB;
      for (int r0 = 0; r0 < n; r0 += 16) {
        const int row = r0 + (t64 >> 2);
        uint4 val[PER];
#pragma unroll
        for (int c = 0; c < PER; ++c) val[c] = make_uint4(0, 0, 0, 0);
        if (row < rows) {
          const int qn = plan[a.off_tq + x.tq_off + (row >> g_shift)];
          const uint4 *src = reinterpret_cast<const uint4 *>(
              q + ((static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (row & (G - 1))) * D) + part * PER;
#pragma unroll
          for (int c = 0; c < PER; ++c) val[c] = __ldg(src + c);
        }
        uint32_t m2 = 0;
#pragma unroll
        for (int c = 0; c < PER; ++c)
          m2 = __vmaxu2(__vmaxu2(m2, val[c].x & 0x7fff7fffu),
                        __vmaxu2(__vmaxu2(val[c].y & 0x7fff7fffu, val[c].z & 0x7fff7fffu), val[c].w & 0x7fff7fffu));
        m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, 1));
        m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, 2));
        if (r0 == 0 && !warp_wait_or_abort(bar + 8 * (L::B_QFREE + qb), ((uc / L::QB) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
        // A row's first reference; NaN spoils a row whose query is not finite.  The softmax reads it with the unit's first tile.
        // The place of unit uc is written again for unit uc + 4, after the last Q.K^T of unit uc + 4 - QB, whose first tile is at least
        // two behind unit uc's, so that its scores' buffer has been given back by the softmax of unit uc's first tile.
        if (part == 0)
          init_s[(uc % U_INIT) * NMAX + row] = row >= rows ? 0.f : (m2 & 0xffffu) >= 0x7f80u || m2 >= 0x7f800000u ? NAN : R_UNSET;
        uint8_t *dst = sm + L::OFF_Q + qb * L::Q_BYTES + (row >> 3) * 1024 + (row & 7) * 128;
#pragma unroll
        for (int c = 0; c < PER; ++c) {
          const int chunk = part * PER + c;
          *reinterpret_cast<uint4 *>(dst + (chunk >> 3) * (NMAX * 128) + (((chunk & 7) ^ (row & 7)) << 4)) = val[c];
        }
      }
      if (!ok) break;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + 8 * (L::B_QFULL + qb));
    }
  } else if (warp < 8) {
    // ================================================================ K's codes to the A operand: a thread per token
    const int wq = warp & 3;
    const uint32_t lane_addr = static_cast<uint32_t>(wq * 32) << 16;
    const int at = (2 * wq + (lane >> 4)) * L::BLOCK + (lane & 15) * 16;             // this token's 16 bytes of the first group
    const int at_scale = (2 * wq + (lane >> 4)) * L::BLOCK + kv4_k_scales(D) + (lane & 15) * (D / 16);
    uint32_t it = 0;
    bool ok = true;
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    while (ok && next(wk, true, ok, x, ll)) {
      for (int k = x.tile_begin; k < x.tile_end; ++k, ++it) {
        const uint32_t s = it % L::STAGES, kb = it % L::KB;
        if (!warp_wait_or_abort(bar + 8 * (L::B_FULL + s), (it / L::STAGES) & 1, abort_flag, limit)) { ok = false; break; }
        const uint8_t *stage = sm + L::OFF_STAGE + s * L::STAGE_BYTES;
        uint4 c[D / 32];
        uint32_t t[D / 64];
#pragma unroll
        for (int g = 0; g < D / 32; ++g) c[g] = *reinterpret_cast<const uint4 *>(stage + at + g * 256);
        if constexpr (D == 128) {
          const uint2 v = *reinterpret_cast<const uint2 *>(stage + at_scale);
          t[0] = v.x; t[1] = v.y;
        } else {
          t[0] = *reinterpret_cast<const uint32_t *>(stage + at_scale);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + 8 * (L::B_EMPTY + s));
        if (!warp_wait_or_abort(bar + 8 * (L::B_KFREE + kb), ((it / L::KB) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          uint32_t o[32];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint32_t t2 = __byte_perm(t[h], t[h], g ? 0x3232 : 0x1010), c2 = kv4_offset_of(t2);
            const uint32_t w[4] = {c[2 * h + g].x, c[2 * h + g].y, c[2 * h + g].z, c[2 * h + g].w};
#pragma unroll
            for (int i = 0; i < 16; ++i) o[16 * g + i] = kv4_value(kv4_pair(w[i >> 2], i & 3), t2, c2);
          }
          tmem_st32_u32(tmem + lane_addr + L::COL_K + kb * L::KW + h * 32, o);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + 8 * (L::B_KFULL + kb));
      }
    }
  } else if (warp < 12) {
    // ================================================================ V's codes to the A operand: a thread per channel
    const int wq = warp & 3;
    const uint32_t lane_addr = static_cast<uint32_t>(wq * 32) << 16;
    const int channel = (wq * 32 + lane) % D, page0 = D == 128 ? 0 : 4 * (wq >> 1);        // first page of this thread's
    const int at = page0 * L::BLOCK + kv4_v_codes(D) + channel * 8, at_scale = page0 * L::BLOCK + kv4_v_scales(D) + (channel / kKv4Group) * 32;
    uint32_t it = 0;
    bool ok = true;
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    while (ok && next(wk, true, ok, x, ll)) {
      for (int k = x.tile_begin; k < x.tile_end; ++k, ++it) {
        const uint32_t s = it % L::STAGES, vb = it % L::VB;
        if (!warp_wait_or_abort(bar + 8 * (L::B_FULL + s), (it / L::STAGES) & 1, abort_flag, limit)) { ok = false; break; }
        if (!warp_wait_or_abort(bar + 8 * (L::B_VFREE + vb), ((it / L::VB) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
        tc_fence_after();
        const uint8_t *stage = sm + L::OFF_STAGE + s * L::STAGE_BYTES;
#pragma unroll
        for (int h = 0; h < L::VW / 32; ++h) {        // four pages at a time
          uint32_t o[32];
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint8_t *block = stage + (4 * h + p) * L::BLOCK;
            const uint2 c = *reinterpret_cast<const uint2 *>(block + at);
            const uint4 ta = *reinterpret_cast<const uint4 *>(block + at_scale), tb = *reinterpret_cast<const uint4 *>(block + at_scale + 16);
            const uint32_t t[8] = {ta.x, ta.y, ta.z, ta.w, tb.x, tb.y, tb.z, tb.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
              o[8 * p + i] = kv4_value(kv4_pair(i < 4 ? c.x : c.y, i & 3), t[i], kv4_offset_of(t[i]));
          }
          if (h == L::VW / 32 - 1) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar + 8 * (L::B_EMPTY + s));
          }
          tmem_st32_u32(tmem + lane_addr + L::COL_V + vb * L::VW + h * 32, o);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar + 8 * (L::B_VFULL + vb));
      }
    }
  } else {
    // ================================================================ softmax + epilogue (2 groups of 128 threads)
    const int grp = (warp - 12) >> 2;             // this group's rows: 8 (2 c + grp) .. + 7 for c = 0, 1, ...
    const int wq = warp & 3, token = wq * 32 + lane;
    const int gt = token;                         // thread of the group
    const uint32_t lane_addr = static_cast<uint32_t>(wq * 32) << 16;
    float *ref_s = reinterpret_cast<float *>(sm + L::OFF_REF), *fact_s = reinterpret_cast<float *>(sm + L::OFF_FACT);
    float *warp_s = reinterpret_cast<float *>(sm + L::OFF_WARP);
    volatile int *vote_s = reinterpret_cast<volatile int *>(sm + L::OFF_VOTE) + 4 * grp;
    const float cap = pv.softcap_log2;
    constexpr bool kKeep = L::CHUNKS <= 4;        // a tile's scores stay in registers from the vote to the weights
    constexpr int SC = kKeep ? L::CHUNKS : 1;
    uint32_t it = 0, uc = 0, meets = 0;
    bool ok = true;
    // the group's four warps meet
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + 8 * (L::B_SYNC + grp));
      return warp_wait_or_abort(bar + 8 * (L::B_SYNC + grp), meets++ & 1, abort_flag, limit);
    };
    Walk wk{0, u0, 0};
    UnitInfo x;
    int ll = 0;
    for (; ok && next(wk, true, ok, x, ll); ++uc) {
      const int nt = x.tile_end - x.tile_begin;
      const int rows = x.n_threads << g_shift, n = rows16(x);
      const uint32_t ob = uc % L::OB;
      const bool fin = x.final_rows != 0;
      const int n_chunks = max(0, (((rows + 7) >> 3) - grp + 1) >> 1);      // of this group
      const int my_row = ((gt >> 3) * 2 + grp) * 8 + (gt & 7);               // the row this thread looks after between tiles
      const bool keeper = my_row < n && gt < NMAX / 2;
      float l[L::CHUNKS][8];
#pragma unroll
      for (int c = 0; c < L::CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) l[c][j] = 0.f;
      for (int k = 0; k < nt; ++k, ++it) {
        const uint32_t sb = it % L::SB, pb = it & 1;
        const uint32_t s_addr = tmem + lane_addr + L::COL_S + sb * NMAX + grp * 8;
        if (!warp_wait_or_abort(bar + 8 * (L::B_SFULL + sb), (it / L::SB) & 1, abort_flag, limit)) { ok = false; break; }
        tc_fence_after();
        if (k == 0) {
          if (keeper) ref_s[my_row] = init_s[(uc % U_INIT) * NMAX + my_row];
          if (!meet()) { ok = false; break; }
        }
        // which rows see this token: bit j of seen[c] for row j of chunk c; pages that every thread sees in full need no look
        const int meta = meta_s[(it % U_RING) * PASTA_TILE_PAGES + (token >> 4)];
        const bool masked = __any_sync(0xffffffffu, meta < 0 || !(meta & PASTA_PMETA_ALL_VISIBLE));
        uint32_t seen[(L::CHUNKS + 3) / 4];
        if (masked) {
#pragma unroll
          for (int i = 0; i < (L::CHUNKS + 3) / 4; ++i) seen[i] = 0;
          const int pos = PASTA_PMETA_PAGE(meta) * PASTA_PAGE + (token & 15);
          const int32_t *vis = plan + a.off_vis + x.vis_off + (meta < 0 ? 0 : PASTA_PMETA_STREAM(meta));
#pragma unroll
          for (int c = 0; c < L::CHUNKS; ++c) {
            if (c >= n_chunks) continue;
            for (int j = 0; j < 8; j += G) {
              const int thread = min((8 * (2 * c + grp) + j) >> g_shift, x.n_threads - 1);
              if (meta >= 0 && pos < vis[thread * x.n_streams]) seen[c >> 2] |= ((1u << G) - 1) << (8 * (c & 3) + j);
            }
          }
        }
        // scores of chunk c in log2 units (capped ones), or what is still to be multiplied by the scale
        auto scores = [&](int c, uint32_t *r) { tmem_ld8_issue(s_addr + c * 16, r); };
        auto finish = [&](int c, float *v) {      // scaled, capped, masked
          if (kCap) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= a.scale_log2 * a.cap_inv;
            softcap_columns<8>(v, cap, true);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= a.scale_log2;
          }
          if (masked) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (!((seen[c >> 2] >> (8 * (c & 3) + j)) & 1)) v[j] = -INFINITY;
          }
        };
        // relative to the references, masked ones -inf
        auto relative = [&](int c, float *v) {
          const float4 r0 = *reinterpret_cast<const float4 *>(ref_s + (2 * c + grp) * 8), r1 = *reinterpret_cast<const float4 *>(ref_s + (2 * c + grp) * 8 + 4);
          if (kCap) {
            finish(c, v);
            v[0] += r0.x; v[1] += r0.y; v[2] += r0.z; v[3] += r0.w; v[4] += r1.x; v[5] += r1.y; v[6] += r1.z; v[7] += r1.w;
          } else {
            fma2v(v[0], v[1], v[0], v[1], a.scale_log2, r0.x, r0.y);
            fma2v(v[2], v[3], v[2], v[3], a.scale_log2, r0.z, r0.w);
            fma2v(v[4], v[5], v[4], v[5], a.scale_log2, r1.x, r1.y);
            fma2v(v[6], v[7], v[6], v[7], a.scale_log2, r1.z, r1.w);
            if (masked) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (!((seen[c >> 2] >> (8 * (c & 3) + j)) & 1)) v[j] = -INFINITY;
            }
          }
        };
        float v[SC][8];
        float top = -INFINITY;
        if constexpr (kKeep) {
#pragma unroll
          for (int c = 0; c < SC; ++c)
            if (c < n_chunks) scores(c, reinterpret_cast<uint32_t *>(v[c]));
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int c = 0; c < SC; ++c) tmem_ld_order8(reinterpret_cast<uint32_t *>(v[c]));
#pragma unroll
          for (int c = 0; c < SC; ++c)
            if (c < n_chunks) {
              relative(c, v[c]);
#pragma unroll
              for (int j = 0; j < 8; ++j) top = fmaxf(top, v[c][j]);
            }
        } else {
#pragma unroll 1
          for (int c = 0; c < n_chunks; ++c) {
            scores(c, reinterpret_cast<uint32_t *>(v[0]));
            tmem_ld_wait8(reinterpret_cast<uint32_t *>(v[0]));
            relative(c, v[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, v[0][j]);
          }
        }
        // ---- the vote.  The word of tile it + 2 is cleared now: everybody has looked at that of tile it - 2, which is the same.
        if (top > R_SLACK) vote_s[it & 3] = 1;
        if (gt == 0) vote_s[(it + 2) & 3] = 0;
        if (!meet()) { ok = false; break; }
        if (vote_s[it & 3] != 0) {
          // ---- some row's reference goes up: maxima of all rows over the tile, then O and l brought to the new references
#pragma unroll 1
          for (int c = 0; c < n_chunks; ++c) {
            float y[8];
            scores(c, reinterpret_cast<uint32_t *>(y));
            tmem_ld_wait8(reinterpret_cast<uint32_t *>(y));
            finish(c, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float m = warp_max(y[j]);
              if (lane == 0) warp_s[wq * NMAX + (2 * c + grp) * 8 + j] = m;
            }
          }
          if (!meet()) { ok = false; break; }
          if (keeper) {
            const float m = fmaxf(fmaxf(warp_s[my_row], warp_s[NMAX + my_row]), fmaxf(warp_s[2 * NMAX + my_row], warp_s[3 * NMAX + my_row]));
            const float old = ref_s[my_row];
            float f = 1.f;
            if (m > -INFINITY && (old == R_UNSET || m + old > R_SLACK)) {
              f = old == R_UNSET ? 0.f : fast_exp2(-old - m);          // (a row that has seen nothing has nothing to bring along)
              ref_s[my_row] = -m;
            }
            fact_s[my_row] = f;
          }
          if (!meet()) { ok = false; break; }
          if (k > 0) {
            // the accumulator is quiet once the P.V of the previous tile has finished
            if (!warp_wait_or_abort(bar + 8 * (L::B_PFREE + ((it - 1) & 1)), ((it - 1) >> 1) & 1, abort_flag, limit)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < L::CHUNKS; ++c) {
              if (c >= n_chunks) continue;
              float f[8];
              bool any = false;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                f[j] = fact_s[(2 * c + grp) * 8 + j];
                any = any || f[j] != 1.f;
                l[c][j] *= f[j];
              }
              if (!any) continue;
#pragma unroll
              for (int w = 0; w < L::OW; ++w) {
                uint32_t o[8];
                const uint32_t at = tmem + lane_addr + L::COL_O + ob * L::OW * NMAX + w * n + (2 * c + grp) * 8;
                tmem_ld8_issue(at, o);
                tmem_ld_wait8(o);
                // a factor of 0 replaces: what no weight has reached yet is 0 times finite numbers, or of a row that is NaN anyway
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f[j]);
                tmem_st8(at, o);
              }
            }
            tmem_st_wait();
          }
          if constexpr (kKeep) {                 // the scores anew, relative to the new references
#pragma unroll
            for (int c = 0; c < SC; ++c)
              if (c < n_chunks) scores(c, reinterpret_cast<uint32_t *>(v[c]));
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
            for (int c = 0; c < SC; ++c) tmem_ld_order8(reinterpret_cast<uint32_t *>(v[c]));
#pragma unroll
            for (int c = 0; c < SC; ++c)
              if (c < n_chunks) relative(c, v[c]);
          }
        }
        // ---- weights: rounded to bf16, summed as rounded, and stored as rows of the B operand
        if constexpr (kKeep) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar + 8 * (L::B_SFREE + sb));
        }
        if (!warp_wait_or_abort(bar + 8 * (L::B_PFREE + pb), ((it >> 1) & 1) ^ 1, abort_flag, limit)) { ok = false; break; }
        const int kr = D == 128 ? token : token & 63;                          // row of the operand
        const int col0 = D == 128 ? 0 : (token >> 6) * (n >> 3);               // its first chunk of 8 columns
        uint8_t *p_row = sm + L::OFF_P + pb * L::P_BYTES + (kr >> 3) * (L::ATOMS * 1024) + (kr & 7) * 128;
#pragma unroll
        for (int c = 0; c < L::CHUNKS; ++c) {
          if (c >= n_chunks) continue;
          float *y = v[kKeep ? c : 0];
          if constexpr (!kKeep) {
            scores(c, reinterpret_cast<uint32_t *>(y));
            tmem_ld_wait8(reinterpret_cast<uint32_t *>(y));
            relative(c, y);
          }
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] = pack_bf16(fast_exp2(y[2 * j]), fast_exp2(y[2 * j + 1]));
            add2(l[c][2 * j], l[c][2 * j + 1], bf16_lo(w[j]), bf16_hi(w[j]));
          }
          const int col = col0 + 2 * c + grp;
          *reinterpret_cast<uint4 *>(p_row + (col >> 3) * 1024 + (((col & 7) ^ (kr & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (!kKeep) mbar_arrive(bar + 8 * (L::B_SFREE + sb));
          mbar_arrive(bar + 8 * (L::B_PFULL + pb));
        }
      }
      if (!ok) break;

      // ---- epilogue: sums over the tokens, then the rows of O, a thread per channel
#pragma unroll
      for (int c = 0; c < L::CHUNKS; ++c) {
        if (c >= n_chunks) continue;
        const float t = warp_sum8(l[c], lane);
        if ((lane & 3) == 0) warp_s[wq * NMAX + (2 * c + grp) * 8 + (lane >> 2)] = t;
      }
      if (!meet()) { ok = false; break; }
      int qn = 0;
      if (keeper) {
        const float sum = (warp_s[my_row] + warp_s[NMAX + my_row]) + (warp_s[2 * NMAX + my_row] + warp_s[3 * NMAX + my_row]);
        const bool spoilt = sum != sum;
        const float m = spoilt ? not_a_row().x : sum > 0.f ? -ref_s[my_row] : -INFINITY, l_all = spoilt ? not_a_row().y : sum;
        fact_s[my_row] = spoilt ? NAN : fin ? (sum > 0.f ? 1.f / sum : 0.f) : 1.f;
        if (my_row < rows) {
          if (!fin) {
            pv.part_ml[static_cast<int64_t>(ll) * pv.rows_per_layer + x.row_base + my_row] = make_float2(m, l_all);
          } else if (a.lse) {
            qn = plan[a.off_tq + x.tq_off + (my_row >> g_shift)];
            a.lse[(static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + x.g * G + (my_row & (G - 1))] = (m + log2f(l_all)) * 0.6931471805599453f;
          }
        }
      }
      if (!meet() || !warp_wait_or_abort(bar + 8 * (L::B_OFULL + ob), (uc / L::OB) & 1, abort_flag, limit)) { ok = false; break; }
      tc_fence_after();
      const uint32_t o_addr = tmem + lane_addr + L::COL_O + ob * L::OW * NMAX + (D == 64 ? (wq >> 1) * n : 0) + grp * 8;
      float *sum_s = reinterpret_cast<float *>(sm + L::OFF_SUM) + (token & 63);
      if constexpr (D == 64) {
        if (wq >= 2) {
#pragma unroll 1
          for (int c = 0; c < n_chunks; ++c) {
            uint32_t o[8];
            tmem_ld8_issue(o_addr + c * 16, o);
            tmem_ld_wait8(o);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum_s[((2 * c + grp) * 8 + j) * 64] = __uint_as_float(o[j]);
          }
        }
        if (!meet()) { ok = false; break; }
      }
      if (D == 128 || wq < 2) {
#pragma unroll 1
        for (int c = 0; c < n_chunks; ++c) {
          uint32_t o[8];
          tmem_ld8_issue(o_addr + c * 16, o);
          tmem_ld_wait8(o);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int row = (2 * c + grp) * 8 + j;
            if (row >= rows) continue;
            const float f = fact_s[row];
            float y = __uint_as_float(o[j]);
            if (D == 64) y += sum_s[row * 64];
            y = f == 0.f ? 0.f : y * f;                // a final row that saw nothing is written as zeros
            if (fin) {
              const int row_q = plan[a.off_tq + x.tq_off + (row >> g_shift)];
              const int64_t at = ((static_cast<int64_t>(ll) * a.n_queries + row_q) * pv.n_q_heads + x.g * G + (row & (G - 1))) * D + token;
              if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
              else static_cast<float *>(a.out)[at] = y;
            } else {
              pv.part_o[(static_cast<int64_t>(ll) * pv.rows_per_layer + x.row_base + row) * D + token] = y;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar + 8 * (L::B_OFREE + ob));
    }
  }

  // ---- tear-down
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // see attn_tensor.cu: what is still in flight for this CTA (bulk copies, MMAs) ends on its own and is waited for
    if (warp == 0 && lane == 0) {
      for (uint32_t j = (prod_it > L::STAGES ? prod_it - L::STAGES : 0); j < prod_it; ++j)
        mbar_wait_bounded(bar + 8 * (L::B_FULL + j % L::STAGES), (j / L::STAGES) & 1);
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

template <int D, int NMAX>
cudaError_t launch_t(const PoolView &pv, const PlanHeader &h, const TensorArgs &a, const void *q, cudaStream_t st) {
  static uint64_t prepared[2] = {0, 0};
  const bool cap = pv.softcap_log2 > 0.f;
  const auto kernel = cap ? attn_kv4_kernel<D, NMAX, true> : attn_kv4_kernel<D, NMAX, false>;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void *>(kernel), U<D, NMAX>::SMEM_BYTES, &prepared[cap]);
  if (e != cudaSuccess) return e;
  return launch_overlapped(kernel, dim3(h.w[PH_T_GRID]), dim3(U_THREADS), U<D, NMAX>::SMEM_BYTES, st, pv, a, static_cast<const __nv_bfloat16 *>(q));
}

template <int D>
cudaError_t launch_d(const PoolView &pv, const PlanHeader &h, const TensorArgs &a, const void *q, cudaStream_t st) {
  const int rows = h.w[PH_T_MAX_ROWS];
  const auto launch = rows <= 16 ? launch_t<D, 16> : rows <= 32 ? launch_t<D, 32> : rows <= 64 ? launch_t<D, 64>
                    : rows <= 96 ? launch_t<D, 96> : launch_t<D, 128>;
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
  a.off_dunit = h.w[PH_OFF_DUNIT]; a.n_dunits = h.w[PH_N_DUNITS];
  a.n_queries = h.w[PH_N_QUERIES]; a.layer_begin = layer_begin; a.layer_count = layer_count;
  a.scale_log2 = scale_log2;
  a.cap_inv = pv.softcap_log2 > 0.f ? 1.f / pv.softcap_log2 : 0.f;
  a.out = out; a.lse = lse; a.out_bf16 = out_bf16 ? 1 : 0;
  return pv.head_dim == 128 ? launch_d<128>(pv, h, a, q, st) : launch_d<64>(pv, h, a, q, st);
}

}  // namespace pasta
