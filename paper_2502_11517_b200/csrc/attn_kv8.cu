// K2 of an 8-bit pool: split-K decode attention over e4m3 codes with one scale per (page, kv head).
//
//   s[r, j]  = q_r . (2^ek Kcode_j) * scale                     (optionally capped: C tanh(s / C))
//   p'[r, j] = 2^(s log2e + ev - ref_r)                         ev: the scale exponent of the page's V, folded into the weight
//   O_r     += p'[r, j] Vcode_j          l_r += p'[r, j] 2^-ev      out = O / l
//
// Folding ev into the exponent makes p' the size of the token's contribution, so the running reference ref_r (raised only
// when exceeded by more than 2^8) bounds what goes through fp16, whatever the pages' scales are.
//
// What bounds it: bytes.  A page of one kv head is 32 D bytes (4 KB at D = 128), which an SM gets in about 176 cycles of
// the measured copy bandwidth.  Codes become fp16 exactly (cvt e4m3x2, 2 cycles per warp and scheduler), so Q.K^T and P.V
// are fp16 mma.sync with fp32 sums: 32 per page for 16 rows, 8 cycles each per scheduler, 64 cycles per page and SM; the
// rows of a request (threads x group) are 4 to 36 in the usual steps.  tcgen05 would need the codes converted back into
// shared memory, or 8-bit weights.
//
// One CTA per (unit, layer, block of 16 MT rows), four warps.  Warp w takes pages w, w + 4, ... of the unit, each through a
// ring of its own that lane 0 fills with one bulk copy per page, so warps never wait for one another inside a unit; each
// keeps its own ref, l and O, which are joined through shared memory at the unit's end.  Three CTAs fit an SM: one's
// start and end are hidden behind the others' copies.  Layouts: token rows of a block are assigned to the columns of the
// score tile in such an order (token 4t + 2j + i of the page is column 2t + i of tile j) that the score accumulators of a
// thread are, rounded to fp16, its A operand of P.V, and V's codes reach the B operand by one transposing 8-bit ldmatrix.
#include <cuda_fp16.h>

#include "device_common.cuh"
#include "kernels.hpp"

namespace pasta {

namespace {

constexpr int E_WARPS = 4, E_THREADS = 32 * E_WARPS;
constexpr int E_STAGES = 4;

struct Kv8Args {
  int32_t off_tunit, off_pages, off_pmeta, off_vis, off_tq;
  int32_t n_queries, layer_begin, row_blocks;
  float scale_log2;
  void *out;                        // [layer_count, n_queries, Hq, D], fp32 or bf16: rows of final units go here
  float *lse;                       // [layer_count, n_queries, Hq] or null
  int32_t out_bf16;
};

template <int D, int MT>
struct Kv8Smem {
  static constexpr int BLOCK = kv8_block_bytes(D);
  static constexpr int KS = D / 16;                                  // k-steps of Q.K^T
  static constexpr int RING = E_WARPS * E_STAGES * BLOCK;            // also the warps' O at the unit's end
  static constexpr int O_BYTES = 16 * MT * D * 4;                    // per warp
  static constexpr int MAIN = RING > E_WARPS * O_BYTES ? RING : E_WARPS * O_BYTES;
  static constexpr int Q_BYTES = MT * KS * 512;                      // fp16 A fragments, 16 bytes per lane
  static constexpr int OFF_Q = MAIN;
  static constexpr int OFF_C1 = OFF_Q + Q_BYTES;                     // per row: scale * log2e / (factor on its Q)
  static constexpr int OFF_ML = OFF_C1 + 16 * MT * 4;                // per warp and row: (ref, l)
  static constexpr int OFF_BAR = OFF_ML + E_WARPS * 16 * MT * 8;
  static constexpr int TOTAL = OFF_BAR + E_WARPS * E_STAGES * 8 + 16;
};

__device__ __forceinline__ void mma_f16(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two 16 x 16 tiles of bytes (lane i < 16: row i of the first, lane 16 + i: row i of the second), transposed: lane
// (g, t) = (lane / 4, lane % 4) gets rows 4t .. 4t + 3 of columns g (r0), g + 8 (r1), and of the second tile (r2, r3)
__device__ __forceinline__ void ldmatrix_t8(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int D, int MT, bool kCap>
__global__ void __launch_bounds__(E_THREADS, MT == 1 ? 3 : 2)
attn_kv8_kernel(PoolView pv, Kv8Args a, const __nv_bfloat16 *__restrict__ q) {
  using S = Kv8Smem<D, MT>;
  constexpr int KS = S::KS, NT = D / 8;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gq = lane >> 2, tq = lane & 3;                        // row / column group of this lane in an MMA fragment
  const int G = pv.n_q_heads / pv.n_kv_heads;
  const int g_shift = 31 - __clz(G);                              // G is 1, 2, 4 or 8
  const int ll = blockIdx.y;
  uint8_t *ring = smem + warp * (E_STAGES * S::BLOCK);
  const uint32_t bar0 = smem_u32(smem + S::OFF_BAR) + warp * E_STAGES * 8;
  float *c1_s = reinterpret_cast<float *>(smem + S::OFF_C1);
  float2 *ml_s = reinterpret_cast<float2 *>(smem + S::OFF_ML);
  if (lane == 0) {
    for (int s = 0; s < E_STAGES; ++s) mbar_init(bar0 + 8 * s, 1);
    mbar_init_fence();
    fence_proxy_async();
  }
  grid_dependency_wait();
  grid_launch_dependents();

  const int4 *U = reinterpret_cast<const int4 *>(pv.plan + a.off_tunit + (blockIdx.x / a.row_blocks) * PU_WORDS);
  const int4 u0 = U[0], u1 = U[1], u2 = U[2];
  const int head = u0.y, rows = u1.w << g_shift;
  const int row0 = (blockIdx.x % a.row_blocks) * (16 * MT);     // a unit's row blocks are neighbours: they share its pages in L2
  if (row0 >= rows) return;
  const int page_begin = u0.z * PASTA_TILE_PAGES, page_end = min(u0.w * PASTA_TILE_PAGES, u1.z);
  const int32_t *pages = pv.plan + a.off_pages + u1.y + page_begin + warp;     // this warp's i-th page: index E_WARPS * i
  const int32_t *metas = pv.plan + a.off_pmeta + u1.y + page_begin + warp;
  const int span = page_end - page_begin - warp;
  const int n_pg = span > 0 ? (span + E_WARPS - 1) / E_WARPS : 0;
  const int n_streams = u2.x, vis_off = u2.y, tq_off = u2.z;
  const bool fin = u2.w != 0;
  const uint8_t *kv_layer = pv.kv_base + (a.layer_begin + ll) * pv.layer_stride;
  const uint16_t *scales = reinterpret_cast<const uint16_t *>(kv_layer + pv.scale_off);

  // page ids, metas and scales of 32 pages live in registers, one per lane; the next 32 are on their way
  auto load_page = [&](int i) {
    int page = i < n_pg ? pages[E_WARPS * i] : 0;
    if (page < 0 || page >= pv.n_pages) { report(pv.status, PASTA_ERR_DEVICE_CHECK); page = 0; }
    return page;
  };
  auto load_scale = [&](int page) { return static_cast<int>(scales[static_cast<int64_t>(page) * pv.n_kv_heads + head]); };
  int cur_page = load_page(lane), nxt_page = load_page(32 + lane);
  int cur_meta = lane < n_pg ? metas[E_WARPS * lane] : 0;
  auto issue = [&](int i, int page) {                               // page: of page i, in lane i % 32's register
    const int p = __shfl_sync(0xffffffffu, page, i & 31);
    if (lane == 0) {
      const int s = i % E_STAGES;
      fence_proxy_async();                                          // the lanes' reads of this stage come before its refill
      mbar_expect_tx(bar0 + 8 * s, S::BLOCK);
      bulk_g2s(smem_u32(ring + s * S::BLOCK), kv_layer + (static_cast<int64_t>(p) * pv.n_kv_heads + head) * S::BLOCK, S::BLOCK,
               bar0 + 8 * s);
    }
  };
  __syncwarp();
  for (int i = 0; i < E_STAGES && i < n_pg; ++i) issue(i, cur_page);
  int cur_sc = load_scale(cur_page), nxt_sc = 0, nxt_meta = 0;

  // ---- the block's query rows as fp16 A fragments.  A row is multiplied by a power of two that brings its largest
  // magnitude to [2^7, 2^8): bf16 numbers then fit fp16 exactly, down to 2^-22 of the row's largest.
  for (int r = warp; r < 16 * MT; r += E_WARPS) {
    const int row = row0 + r;
    constexpr int E = D / 32;                                       // elements per lane
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
    if (row < rows) {
      const int qn = pv.plan[a.off_tq + tq_off + (row >> g_shift)];
      const __nv_bfloat16 *src = q + ((static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + head * G + (row & (G - 1))) * D + lane * E;
      if (E == 4) {
        const uint2 w = *reinterpret_cast<const uint2 *>(src);
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[E - 2] = bf16_lo(w.y); x[E - 1] = bf16_hi(w.y);
      } else {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(src);
        x[0] = bf16_lo(w); x[1] = bf16_hi(w);
      }
    }
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) amax = max(amax, __float_as_uint(x[e]) & 0x7fffffffu);
    amax = __reduce_max_sync(0xffffffffu, amax);
    const int up = max(-126, min(126, 7 - (static_cast<int>(amax >> 23) - 127)));
    const float f = pow2f(up);
    // lane's elements: d = lane * E ...; thread t of a fragment owns d in [t D / 4, (t + 1) D / 4), four per k-step
    const int t = lane >> 3, within = (lane & 7) * E, ks = within >> 2;
    uint32_t *frag = reinterpret_cast<uint32_t *>(smem + S::OFF_Q) + (((r >> 4) * KS + ks) * 32 + (r & 7) * 4 + t) * 4 + ((r >> 3) & 1);
    if (E == 4) {
      frag[0] = pack_f16(x[0] * f, x[1] * f);
      frag[2] = pack_f16(x[E - 2] * f, x[E - 1] * f);
    } else {
      frag[(lane & 1) * 2] = pack_f16(x[0] * f, x[1] * f);
    }
    if (lane == 0) c1_s[r] = a.scale_log2 * pow2f(-up);
  }
  __syncthreads();

  uint32_t qf[MT == 1 ? KS : 1][4];
  if (MT == 1) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 v = *reinterpret_cast<const uint4 *>(smem + S::OFF_Q + (ks * 32 + lane) * 16);
      qf[MT == 1 ? ks : 0][0] = v.x; qf[MT == 1 ? ks : 0][1] = v.y; qf[MT == 1 ? ks : 0][2] = v.z; qf[MT == 1 ? ks : 0][3] = v.w;
    }
  }
  float c1[MT][2], ref[MT][2], l[MT][2], o[MT][NT][4];
  int vis_row[MT][2], vis[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = m * 16 + h * 8 + gq;
      c1[m][h] = c1_s[r];
      ref[m][h] = -INFINITY;
      l[m][h] = 0.f;
      vis[m][h] = 0;
      vis_row[m][h] = row0 + r < rows ? a.off_vis + vis_off + ((row0 + r) >> g_shift) * n_streams : -1;
    }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][n][e] = 0.f;
  const float cap = pv.softcap_log2, cap_k2 = kCap ? 2.f * 1.4426950408889634f / cap : 0.f;
  int cur_stream = -1;
  int consumed = 0;
  bool ok = true;

  for (int i = 0; i < n_pg; ++i) {
    if (i > 0 && (i & 31) == 0) {
      cur_page = nxt_page; cur_sc = nxt_sc; cur_meta = nxt_meta;
      nxt_page = load_page(i + 32 + lane);
    }
    if ((i & 31) == 16 && (i & ~31) + 32 < n_pg) {                  // by now the next page ids have arrived
      const int j = (i & ~31) + 32 + lane;
      nxt_sc = load_scale(nxt_page);
      nxt_meta = j < n_pg ? metas[E_WARPS * j] : 0;
    }
    const int s = i % E_STAGES;
    if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar0 + 8 * s, (i / E_STAGES) & 1, pv.wait_limit))) { ok = false; consumed = i; break; }
    const uint8_t *blk = ring + s * S::BLOCK;
    const int sc2 = __shfl_sync(0xffffffffu, cur_sc, i & 31), meta = __shfl_sync(0xffffffffu, cur_meta, i & 31);
    const int ek = static_cast<int8_t>(sc2 & 0xff), ev = static_cast<int8_t>(sc2 >> 8);

    // ---- what each row sees of this page
    const bool all_visible = (meta & PASTA_PMETA_ALL_VISIBLE) != 0;
    int thr[MT][2];
    bool seen = true;
    if (!all_visible) {
      const int stream = PASTA_PMETA_STREAM(meta), first = PASTA_PMETA_PAGE(meta) * PASTA_PAGE;
      bool any = false;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (stream != cur_stream) vis[m][h] = vis_row[m][h] >= 0 ? pv.plan[vis_row[m][h] + stream] : 0;
          thr[m][h] = vis[m][h] - first;
          any = any || thr[m][h] > 0;
        }
      cur_stream = stream;
      seen = __any_sync(0xffffffffu, any);
    }
    if (seen) {
      // ---- scores
      float sc[MT][2][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[m][j][e] = 0.f;
      const int tok = 4 * (gq >> 1) + (gq & 1);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        uint4 kk[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
          kk[j] = *reinterpret_cast<const uint4 *>(blk + kv8_chunk_offset<D>(0, tok + 2 * j, D == 128 ? 2 * tq + h : tq));
        const uint32_t kw[2][4] = {{kk[0].x, kk[0].y, kk[0].z, kk[0].w}, {kk[1].x, kk[1].y, kk[1].z, kk[1].w}};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t b[2][2];
          e4m3x4_to_f16x4(kw[0][w], b[0][0], b[0][1]);
          e4m3x4_to_f16x4(kw[1][w], b[1][0], b[1][1]);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            uint32_t af[4];
            if (MT == 1) {
#pragma unroll
              for (int e = 0; e < 4; ++e) af[e] = qf[MT == 1 ? h * 4 + w : 0][e];
            } else {
              const uint4 v = *reinterpret_cast<const uint4 *>(smem + S::OFF_Q + ((m * KS + h * 4 + w) * 32 + lane) * 16);
              af[0] = v.x; af[1] = v.y; af[2] = v.z; af[3] = v.w;
            }
            mma_f16(sc[m][0], af, b[0][0], b[0][1]);
            mma_f16(sc[m][1], af, b[1][0], b[1][1]);
          }
        }
      }
      // ---- exponents: scaled, capped, masked, the V scale folded in
      const float fk = pow2f(ek), fev = static_cast<float>(ev);
      bool need = false;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float c = c1[m][h] * fk;
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float &x = sc[m][j][2 * h + e];
              if (kCap) x = softcap(x * c, cap, cap_k2) + fev;
              else x = fmaf(x, c, fev);
              if (!all_visible && 4 * tq + 2 * j + e >= thr[m][h]) x = -INFINITY;
              mx = fmaxf(mx, x);
            }
          need = need || mx > ref[m][h] + 8.f;
        }
      if (__any_sync(0xffffffffu, need)) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float mx = fmaxf(fmaxf(sc[m][0][2 * h], sc[m][0][2 * h + 1]), fmaxf(sc[m][1][2 * h], sc[m][1][2 * h + 1]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            if (mx > ref[m][h] + 8.f) {                             // the same answer for the row's four lanes
              const float f = fast_exp2(ref[m][h] - mx);            // 0 the first time
              ref[m][h] = mx;
              l[m][h] *= f;
#pragma unroll
              for (int n = 0; n < NT; ++n) { o[m][n][2 * h] *= f; o[m][n][2 * h + 1] *= f; }
            }
          }
      }
      const float fl = pow2f(-ev);
      uint32_t pa[MT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float rf = ref[m][h] == -INFINITY ? 0.f : ref[m][h];
          const float p0 = fast_exp2(sc[m][0][2 * h] - rf), p1 = fast_exp2(sc[m][0][2 * h + 1] - rf);
          const float p2 = fast_exp2(sc[m][1][2 * h] - rf), p3 = fast_exp2(sc[m][1][2 * h + 1] - rf);
          l[m][h] = fmaf((p0 + p1) + (p2 + p3), fl, l[m][h]);
          // fp16 weights: off by at most 2^-11 of the weight, or 2^-25 of the row's reference; the sum l keeps all bits
          pa[m][h] = pack_f16(p0, p1);
          pa[m][2 + h] = pack_f16(p2, p3);
        }
      // ---- O += P V
      const int vrow = lane & 15;
#pragma unroll
      for (int c = 0; c < D / 16; c += 2) {
        uint32_t v[4];
        ldmatrix_t8(smem_u32(blk) + kv8_chunk_offset<D>(1, vrow, c + (lane >> 4)), v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t b0, b1;
          e4m3x4_to_f16x4(v[k], b0, b1);
#pragma unroll
          for (int m = 0; m < MT; ++m) mma_f16(o[m][2 * c + k], pa[m], b0, b1);
        }
      }
    }
    __syncwarp();                                                   // every lane is done with the stage
    if (i + E_STAGES < n_pg) issue(i + E_STAGES, (i + E_STAGES) / 32 == i / 32 ? cur_page : nxt_page);
  }
  if (!ok) {
    // give up: report, and wait (bounded) for the copies still in flight; the outputs of this launch are undefined
    if (lane == 0) report(pv.status, PASTA_ERR_TIMEOUT);
    for (int j = consumed; j < n_pg && j < consumed + E_STAGES; ++j) mbar_wait_bounded(bar0 + 8 * (j % E_STAGES), (j / E_STAGES) & 1);
  }

  // ---- join the four warps: (ref, l) and O through shared memory (a warp's O takes the place of its own ring)
  static_assert(S::O_BYTES * E_WARPS <= S::MAIN, "O of all warps");
  __syncthreads();                                                  // O regions may reach into a neighbour's ring
  float *o_s = reinterpret_cast<float *>(smem + warp * S::O_BYTES);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = m * 16 + h * 8 + gq;
      float lt = l[m][h];
      lt += __shfl_xor_sync(0xffffffffu, lt, 1);
      lt += __shfl_xor_sync(0xffffffffu, lt, 2);
      if (tq == 0) ml_s[warp * 16 * MT + r] = make_float2(ref[m][h], lt);
      // 8-byte pieces: piece x of a row goes to x ^ (4 (r % 4)) so that the eight rows a warp writes at once spread over the banks
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *reinterpret_cast<float2 *>(o_s + r * D + (((n * 4 + tq) ^ ((r & 3) << 2)) << 1)) = make_float2(o[m][n][2 * h], o[m][n][2 * h + 1]);
    }
  __syncthreads();
  const int live = min(rows - row0, 16 * MT);
  constexpr int PER = D / 4;                                        // threads per row, 4 elements each
  for (int x = tid; x < live * PER; x += E_THREADS) {
    const int r = x / PER, d4 = x % PER;
    float ref_w[E_WARPS], l_w[E_WARPS], m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < E_WARPS; ++w) {
      const float2 ml = ml_s[w * 16 * MT + r];
      ref_w[w] = ml.x; l_w[w] = ml.y;
      m_all = fmaxf(m_all, ml.x);
    }
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < E_WARPS; ++w) {
      if (ref_w[w] == -INFINITY) continue;                          // that warp saw nothing of this row
      const float f = fast_exp2(ref_w[w] - m_all);
      const float4 v = *reinterpret_cast<const float4 *>(smem + w * S::O_BYTES + (r * D + (((d4 * 2) ^ ((r & 3) << 2)) << 1)) * 4);
      l_all = fmaf(f, l_w[w], l_all);
      acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]);
      acc[2] = fmaf(f, v.z, acc[2]); acc[3] = fmaf(f, v.w, acc[3]);
    }
    const int row = row0 + r;
    if (fin) {
      const int qn = pv.plan[a.off_tq + tq_off + (row >> g_shift)];
      const int64_t orow = (static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + head * G + (row & (G - 1));
      const float inv = l_all > 0.f ? 1.f / l_all : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= inv;
      if (a.out_bf16) {
        const __nv_bfloat162 b0 = __floats2bfloat162_rn(acc[0], acc[1]), b1 = __floats2bfloat162_rn(acc[2], acc[3]);
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + orow * D + d4 * 4) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&b0), *reinterpret_cast<const uint32_t *>(&b1));
      } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + orow * D + d4 * 4) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      }
      if (a.lse && d4 == 0) a.lse[orow] = (m_all + log2f(l_all)) * 0.6931471805599453f;
    } else {
      const int64_t prow = static_cast<int64_t>(ll) * pv.rows_per_layer + u1.x + row;
      if (d4 == 0) pv.part_ml[prow] = make_float2(m_all, l_all);
      if (l_all > 0.f) *reinterpret_cast<float4 *>(pv.part_o + prow * D + d4 * 4) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    }
  }
}

template <int D, int MT, bool kCap>
cudaError_t launch_t(const PoolView &pv, const PlanHeader &h, Kv8Args a, int32_t layer_count, const void *q, cudaStream_t st) {
  using S = Kv8Smem<D, MT>;
  static uint64_t prepared = 0;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void *>(attn_kv8_kernel<D, MT, kCap>), S::TOTAL, &prepared);
  if (e != cudaSuccess) return e;
  a.row_blocks = (h.w[PH_T_MAX_ROWS] + 16 * MT - 1) / (16 * MT);
  return launch_overlapped(attn_kv8_kernel<D, MT, kCap>, dim3(h.w[PH_N_TUNITS] * a.row_blocks, layer_count), dim3(E_THREADS), S::TOTAL, st,
                           pv, a, static_cast<const __nv_bfloat16 *>(q));
}

}  // namespace

cudaError_t launch_attn_kv8(const PoolView &pv, const PlanHeader &h, int32_t layer_begin, int32_t layer_count,
                            const void *q, float scale_log2, void *out, float *lse, bool out_bf16, cudaStream_t st) {
  if (h.w[PH_N_TUNITS] == 0 || layer_count == 0) return cudaSuccess;
  const Kv8Args a{h.w[PH_OFF_TUNIT], h.w[PH_OFF_PAGES], h.w[PH_OFF_PMETA], h.w[PH_OFF_VIS], h.w[PH_OFF_TQ],
                  h.w[PH_N_QUERIES], layer_begin, 1, scale_log2, out, lse, out_bf16 ? 1 : 0};
  const bool cap = pv.softcap_log2 > 0.f;
  const int mt = h.w[PH_T_MAX_ROWS] <= 16 ? 1 : 2;
#define PASTA_E(DD, MM, CC) \
  if (pv.head_dim == DD && mt == MM && cap == CC) return launch_t<DD, MM, CC>(pv, h, a, layer_count, q, st);
  PASTA_E(128, 1, false) PASTA_E(128, 1, true) PASTA_E(128, 2, false) PASTA_E(128, 2, true)
  PASTA_E(64, 1, false) PASTA_E(64, 1, true) PASTA_E(64, 2, false) PASTA_E(64, 2, true)
#undef PASTA_E
  return cudaErrorInvalidValue;
}

}  // namespace pasta
