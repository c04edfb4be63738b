// What the tcgen05 attention kernels share: descriptors, MMA and TMEM access, packed arithmetic, bounded waits between
// roles, and a role's walk through its CTA's units.  Included by one source file each; everything has internal linkage.
#pragma once
#include "device_common.cuh"
#include "kernels.hpp"

namespace pasta {

namespace {

constexpr int T_TILE = PASTA_TILE_PAGES * PASTA_PAGE;          // 128 tokens
static_assert(PASTA_TILE_PAGES == 8, "the kernels are written for 8-page tiles");
constexpr int T_RING = 8;                                      // unit records the producer keeps published (64 B each)
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t IDESC_M128 = (128u >> 4) << 24, IDESC_M64 = (64u >> 4) << 24;      // instruction descriptor: rows
constexpr int T_M64_ROWS = 64;

__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(lbo_bytes >> 4) << 16) |
         (static_cast<uint64_t>(sbo_bytes >> 4) << 32) | (1ull << 46) | (2ull << 61);   // version 1, 128-byte swizzle
}

__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A operand from TMEM: row m in lane m, two bf16 per 32-bit column (16 K-elements = 8 columns)
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define PASTA_R32(v) \
  v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15], v[16], v[17], \
  v[18], v[19], v[20], v[21], v[22], v[23], v[24], v[25], v[26], v[27], v[28], v[29], v[30], v[31]

// 32 consecutive fp32 columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
      "%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
  // the wait names the registers so that nothing that uses them can be scheduled above it
  asm volatile("tcgen05.wait::ld.sync.aligned;"
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
        "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
        "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
        "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
      :: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// The same load without its wait, and the wait by itself, so that several loads can be in flight before one wait.  The
// wait (and tmem_ld_order for a second register set) names the registers so that nothing that uses them can be
// scheduled above it.
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
      "%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
#define PASTA_RW32(r)                                                                                                  \
  "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),          \
  "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]),   \
  "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]),  \
  "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
__device__ __forceinline__ void tmem_ld_wait32(uint32_t *r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : PASTA_RW32(r) :: "memory");
}
__device__ __forceinline__ void tmem_ld_order32(uint32_t *r) { asm volatile("" : PASTA_RW32(r) :: "memory"); }
// 16 consecutive fp32 columns, issued without the wait
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
#define PASTA_RW16(r)                                                                                                  \
  "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),          \
  "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
// waits for every load of this thread in flight; names the registers of two of them
__device__ __forceinline__ void tmem_ld_wait16x2(uint32_t *r0, uint32_t *r1) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : PASTA_RW16(r0), PASTA_RW16(r1) :: "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float *v) {
  uint32_t r[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
      "%29,%30,%31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st32_u32(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
      "%29,%30,%31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// two fp32 lanes at once: {x0, x1} = {a0, a1} * {b, b} + {c, c}
__device__ __forceinline__ void fma2(float &x0, float &x1, float a0, float a1, float b, float c) {
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\t"
      "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %5};\n\t"
      "fma.rn.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}
// {x0, x1} = {a0, a1} * {b, b} + {c0, c1}
__device__ __forceinline__ void fma2v(float &x0, float &x1, float a0, float a1, float b, float c0, float c1) {
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\t"
      "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %4};\n\tmov.b64 rc, {%5, %6};\n\t"
      "fma.rn.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b), "f"(c0), "f"(c1));
}
// {s0, s1} += {p0, p1}
__device__ __forceinline__ void add2(float &s0, float &s1, float p0, float p1) {
  asm("{\n\t.reg .b64 ra, rb, rd;\n\t"
      "mov.b64 ra, {%0, %1};\n\tmov.b64 rb, {%2, %3};\n\t"
      "add.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "+f"(s0), "+f"(s1) : "f"(p0), "f"(p1));
}
// {a0, a1} = {a0, a1} * {b0, b1} + {c, c}
__device__ __forceinline__ void horner2(float &a0, float &a1, float b0, float b1, float c) {
  asm("{\n\t.reg .b64 ra, rb, rc;\n\t"
      "mov.b64 ra, {%0, %1};\n\tmov.b64 rb, {%2, %3};\n\tmov.b64 rc, {%4, %4};\n\t"
      "fma.rn.f32x2 ra, ra, rb, rc;\n\tmov.b64 {%0, %1}, ra;\n\t}"
      : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1), "f"(c));
}
// {x0, x1} = {a0, a1} * {b0, b1}
__device__ __forceinline__ void mul2(float &x0, float &x1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 ra, rb, rd;\n\t"
      "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// {x0, x1} = C tanh({x0, x1}) by softcap's polynomial, for magnitudes up to 1: 9 packed operations
__device__ __forceinline__ void softcap_poly2(float &x0, float &x1, float C) {
  float u0, u1, t0 = kTanhPolyTop, t1 = kTanhPolyTop;
  mul2(u0, u1, x0, x1, x0, x1);
#define PASTA_STEP(c) horner2(t0, t1, u0, u1, c);
  PASTA_TANH_POLY(PASTA_STEP)
#undef PASTA_STEP
  mul2(t0, t1, t0, t1, x0, x1);
  mul2(x0, x1, t0, t1, C, C);
}
// x[j] = C tanh(x[j]) for the N scores of every thread of a warp; x = score / C, C in log2 units.
// The form with ex2 and rcp takes two of the special-function unit's slots, 16 cycles per column and warp, on top of the
// weight's one; the exponential units are what bounds a capped tile.  Scores that a cap is meant for mostly lie well inside
// it, so a warp whose scores all have |x| <= 1 takes softcap's polynomial alone (64 responses over a bf16 cache: 162 -> 148 us).
// Otherwise both are worked out and every score takes the one its own size asks for, so that the vote decides on time only: a
// row's capped scores do not depend on the rows beside it or on what its masked columns hold.  Rows that are not active do not
// count.
template <int N>
__device__ __forceinline__ void softcap_columns(float *x, float C, bool active) {
  float m0 = 0.f, m1 = 0.f;
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    m0 = fmaxf(m0, fabsf(x[j]));
    m1 = fmaxf(m1, fabsf(x[j + 1]));
  }
  if (__any_sync(0xffffffffu, active && fmaxf(m0, m1) > 1.f)) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      float y0 = x[j], y1 = x[j + 1];
      softcap_poly2(y0, y1, C);
      x[j] = fabsf(x[j]) > 1.f ? softcap_any(x[j], C) : y0;
      x[j + 1] = fabsf(x[j + 1]) > 1.f ? softcap_any(x[j + 1], C) : y1;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 2) softcap_poly2(x[j], x[j + 1], C);
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Bounded wait of one role for another that also gives up when some role of the CTA has already given up.
__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, volatile int *abort_flag, long long limit) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) { *abort_flag = 1; return false; }
  }
}
// The same for a whole warp whose lanes go on to warp-wide instructions (tcgen05.ld / st, votes, __syncwarp): the
// lanes poll on their own, so the warp takes the decision as one.
__device__ __forceinline__ bool warp_wait_or_abort(uint32_t bar, uint32_t parity, volatile int *abort_flag, long long limit) {
  return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_flag, limit));
}

// bulk copy whose lines are the first to leave L2: every page is read once per launch
__device__ __forceinline__ void bulk_g2s_stream(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
      ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy)
      : "memory");
}

struct UnitInfo {
  int treq, g, tile_begin, tile_end, row_base;
  int page_off, n_pages, n_threads, n_streams, vis_off, tq_off, final_rows;
};

__device__ __forceinline__ UnitInfo load_unit(const int32_t *plan, int off_tunit, int off_treq, int u) {
  (void)off_treq;
  const int4 *U = reinterpret_cast<const int4 *>(plan + off_tunit + u * PU_WORDS);   // tables start 16-byte aligned
  const int4 a = U[0], b = U[1], c = U[2];
  UnitInfo x;
  x.treq = a.x; x.g = a.y; x.tile_begin = a.z; x.tile_end = a.w;
  x.row_base = b.x; x.page_off = b.y; x.n_pages = b.z; x.n_threads = b.w;
  x.n_streams = c.x; x.vis_off = c.y; x.tq_off = c.z; x.final_rows = c.w;
  return x;
}

struct TensorArgs {
  int32_t off_tunit, off_treq, off_tcta, off_pages, off_pmeta, off_vis, off_tq;
  int32_t n_tunits = 0;             // (4-bit pools) units assigned to CTAs in advance, per layer
  int32_t off_dunit, n_dunits;      // units no CTA owns in advance (per layer): taken from a counter at run time
  int32_t n_queries, layer_begin, layer_count;
  float scale_log2;
  float cap_inv;                    // capped scores: 1 / C, C in log2 units
  void *out;                        // [layer_count, n_queries, Hq, 128], fp32 or bf16: rows of final units go here
  float *lse;                       // [layer_count, n_queries, Hq] or null
  int32_t out_bf16;
};

// A role's place in its CTA's sequence of units: first the units assigned to the CTA, layer by layer, whose records every
// role reads from the plan itself; then units of the shared pool (whole short runs kept back by the planner), taken from
// a counter in global memory.  Only the producer, which gets to every unit first, touches the counter: it publishes the
// record (and layer) of each shared unit it takes in a ring of T_RING slots in shared memory, and the other roles read
// the records from there in the same order, without a round trip to global memory at the start of a unit.  A record
// with tile_end = 0 ends the sequence.  The producer is at most its stages' number of tiles, hence units, ahead of the tile whose
// P.V has finished, and no role is a whole unit behind that one when it reads its next record, so a slot is not
// overwritten before everybody has read it.
struct Walk { int ll, u, k; };

template <bool kProducer, bool kShared>
__device__ __forceinline__ bool next_unit(Walk &w, const TensorArgs &a, const int32_t *plan, int u0, int u1, volatile int *ring,
                                          int32_t *counter, int lane, bool whole_warp, volatile int *abort_flag,
                                          long long limit, bool &ok, UnitInfo &x, int &ll) {
  if (u0 < u1 && w.ll < a.layer_count) {
    x = load_unit(plan, a.off_tunit, 0, w.u);
    ll = w.ll;
    if (++w.u == u1) { w.u = u0; ++w.ll; }
    return true;
  }
  if (!kShared) return false;        // this build of the kernel serves plans without shared units
  if (a.n_dunits == 0) return false;
  int32_t *slot = const_cast<int32_t *>(reinterpret_cast<volatile int32_t *>(ring)) + 2 + 16 * (w.k % T_RING);
  if (kProducer) {
    int id = -1;
    if (lane == 0) {
      id = atomicAdd(counter, 1);
      if (id >= a.n_dunits * a.layer_count) id = -1;
    }
    id = __shfl_sync(0xffffffffu, id, 0);
    if (id >= 0) {
      ll = id / a.n_dunits;
      x = load_unit(plan, a.off_dunit, 0, id - ll * a.n_dunits);
    }
    if (lane == 0) {
      int4 *s4 = reinterpret_cast<int4 *>(slot);
      s4[0] = make_int4(x.treq, x.g, x.tile_begin, id >= 0 ? x.tile_end : 0);
      s4[1] = make_int4(x.row_base, x.page_off, x.n_pages, x.n_threads);
      s4[2] = make_int4(x.n_streams, x.vis_off, x.tq_off, ll);
      s4[3] = make_int4(x.final_rows, 0, 0, 0);
      __threadfence_block();
      ring[0] = w.k + 1;
    }
    ++w.k;
    return id >= 0;
  }
  int got = 1;
  if (!whole_warp || lane == 0) {
    if (ring[0] <= w.k) {
      const long long t0 = clock64();
      while (ring[0] <= w.k) {
        if (*abort_flag) { got = 0; break; }
        if (clock64() - t0 > limit) { *abort_flag = 1; got = 0; break; }
        __nanosleep(64);
      }
    }
  }
  if (whole_warp) {
    got = __shfl_sync(0xffffffffu, got, 0);
    __syncwarp();
  }
  if (!got) { ok = false; return false; }
  const int4 *s4 = reinterpret_cast<const int4 *>(slot);
  const int4 ra = s4[0], rb = s4[1], rc = s4[2];
  x.final_rows = s4[3].x;
  ++w.k;
  if (ra.w == 0) return false;
  x.treq = ra.x; x.g = ra.y; x.tile_begin = ra.z; x.tile_end = ra.w;
  x.row_base = rb.x; x.page_off = rb.y; x.n_pages = rb.z; x.n_threads = rb.w;
  x.n_streams = rc.x; x.vis_off = rc.y; x.tq_off = rc.z; ll = rc.w;
  return true;
}

}  // namespace

}  // namespace pasta
