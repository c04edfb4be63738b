// K2 of an 8-bit pool, head_dim 64: split-K decode attention over e4m3 codes with one scale per (page, kv head).
//
//   s[r, j]  = q_r . (2^ek Kcode_j) * scale                     (optionally capped: C tanh(s / C))
//   p'[r, j] = 2^(s log2e + ev - ref_r)                         ev: the scale exponent of the page's V, folded into the weight
//   O_r     += p'[r, j] Vcode_j          l_r += p'[r, j] 2^-ev      out = O / l
//
// Folding ev into the exponent makes p' the size of the token's contribution, so the running reference ref_r (raised only
// when exceeded by more than 2^8) bounds what goes through fp16, whatever the pages' scales are.
//
// What bounds it.  A page of one kv head is 2 KB, which an SM gets in about 88 cycles of the measured copy bandwidth.  Codes
// become fp16 exactly (cvt e4m3x2, 2 cycles per warp and scheduler), Q.K^T and P.V are fp16 mma.sync with fp32 sums (8 cycles
// per m16n8k16): 32 cycles of matrix pipe per page and 16 rows, and several times that of issue, which is what is left:
// 32 requests of 8 to 20 rows, 2 layers, 75 MB: 31.9 us, 38 % of the copy bandwidth, against 12.2 us for the bytes.
// (mma.sync because a row of codes is 64 bytes and the steps have few rows; a tcgen05 form was built at head_dim 128 only, where
// this design took 194, 176 and 449 us for the three cases of attn_kv8_tensor.cu, where that takes 180, 170 and 230.  The e4m3 form of
// mma.sync is slower: 850 instructions per page and 16 rows were counted with it at head_dim 128 against 300 here.)
//
// One CTA of W warps per (unit, layer, group of row tiles).  A row tile is 16 stacked rows; the group's `tiles` row tiles are
// spread over the warps, warp w = lane_of_pages * tiles + tile, so that W / tiles pairs of pages are worked on at a time and
// every page is brought in once for all row tiles of the group.  Pages go, two to a stage, through rings of bulk copies, one
// ring per page lane, the CTA's stages shared out among them.  With one row tile a warp refills its own ring and warps
// never wait for one another inside a unit; with more, the first tile's warp refills a stage once every tile's warp has
// let go of it.  Each warp keeps its own ref, l and O, joined through shared memory at the unit's end.
// W = 2, six CTAs to an SM, when there is work for all of them: the starts and ends of units, chains of a few trips to
// memory, are hidden behind the other CTAs' copies.  W = 6 for small steps, whose runs are units and which only last as
// long as one of them.  Token rows of a page are assigned to the columns of the score tile in such an order (token
// 4t + 2j + i is column 2t + i of tile j) that a thread's score accumulators are, rounded to fp16, its A operand of P.V, and
// V's codes reach the B operand by one transposing 8-bit ldmatrix.
#include <cuda_fp16.h>

#include <type_traits>

#include "device_common.cuh"
#include "kernels.hpp"

namespace pasta {

namespace {

constexpr int D = 64;                      // head_dim
constexpr int E_LAG = 1;                   // stages a shared ring is refilled behind the one being worked on

struct Kv8Args {
  int32_t off_tunit, off_pages, off_pmeta, off_vis, off_tq;
  int32_t n_queries, layer_begin, groups;      // groups: CTAs per unit and layer, enough for the highest unit
  float scale_log2;
  void *out;                        // [layer_count, n_queries, Hq, D], fp32 or bf16: rows of final units go here
  float *lse;                       // [layer_count, n_queries, Hq] or null
  int32_t out_bf16;
};

// Row tiles of one CTA of W warps for a unit of `tiles` row tiles in all.  Two warps take two tiles at most; of six warps
// every size keeps all busy except 5 (five of six).
template <int W>
__host__ __device__ constexpr int kv8_group_tiles(int tiles) {
  if (W == 2) return tiles < 2 ? tiles : 2;
  return tiles <= 3 ? tiles : tiles == 4 ? 2 : tiles == 5 ? 5 : 3;
}
template <int W>
__host__ __device__ constexpr int kv8_max_groups(int tiles) {            // CTAs of any unit of up to that many row tiles
  int most = 1;
  for (int t = 1; t <= tiles; ++t) {
    const int n = (t + kv8_group_tiles<W>(t) - 1) / kv8_group_tiles<W>(t);
    most = n > most ? n : most;
  }
  return most;
}

template <int W>
struct Kv8Smem {
  static constexpr int STAGES = 2 * W;                               // of the CTA, two pages each
  static constexpr int BLOCK = kv8_block_bytes(D);
  static constexpr int O_BYTES = 16 * D * 4;                         // per warp, at the unit's end
  static constexpr int STAGE = 2 * BLOCK;
  static constexpr int RING = STAGES * STAGE;
  static constexpr int OFF_ML = RING > W * O_BYTES ? RING : W * O_BYTES;      // per warp and row: (ref, l)
  static constexpr int OFF_BAR = OFF_ML + W * 16 * 8;                // full[STAGES], empty[STAGES]
  static constexpr int TOTAL = OFF_BAR + 2 * STAGES * 8;
};

__device__ __forceinline__ void mma_f16(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same with nothing to add to
__device__ __forceinline__ void mma_f16_first(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// two 16 x 16 tiles of bytes (lane i < 16: row i of the first, lane 16 + i: row i of the second), transposed: lane
// (g, t) = (lane / 4, lane % 4) gets rows 4t .. 4t + 3 of columns g (r0), g + 8 (r1), and of the second tile (r2, r3)
__device__ __forceinline__ void ldmatrix_t8(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int W, bool kCap>
__global__ void __launch_bounds__(32 * W, 12 / W)
attn_kv8_kernel(PoolView pv, Kv8Args a, const __nv_bfloat16 *__restrict__ q) {
  using S = Kv8Smem<W>;
  constexpr int KS = D / 16, NT = D / 8;                          // k-steps of Q.K^T, output tiles of P.V
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gq = lane >> 2, tq = lane & 3;                        // row / column group of this lane in an MMA fragment
  const int G = pv.n_q_heads / pv.n_kv_heads;
  const int g_shift = 31 - __clz(G);                              // G is 1, 2, 4 or 8
  const int ll = blockIdx.y;
  const uint32_t smem_base = smem_u32(smem);
  const uint32_t bars = smem_base + S::OFF_BAR;
  float2 *ml_s = reinterpret_cast<float2 *>(smem + S::OFF_ML);
  grid_dependency_wait();
  grid_launch_dependents();

  const int4 *U = reinterpret_cast<const int4 *>(pv.plan + a.off_tunit + (blockIdx.x / a.groups) * PU_WORDS);
  const int4 u0 = U[0], u1 = U[1], u2 = U[2];
  const int head = u0.y, rows = u1.w << g_shift;
  const int all_tiles = (rows + 15) >> 4;
  const int tile0 = (blockIdx.x % a.groups) * kv8_group_tiles<W>(all_tiles);      // a unit's groups are neighbours: they share its pages in L2
  if (tile0 >= all_tiles) return;
  const int tiles = min(kv8_group_tiles<W>(all_tiles), all_tiles - tile0);
  const int lanes = W / tiles;                              // page lanes
  const int stages = S::STAGES / lanes;                            // of one lane's ring
  const int plane = warp / tiles, tile = warp - plane * tiles;
  const bool works = plane < lanes;
  const bool shared_ring = tiles > 1, producer = tile == 0;
  if (tid < S::STAGES) {
    mbar_init(bars + 8 * tid, 1);
    mbar_init(bars + 8 * (S::STAGES + tid), tiles);
    mbar_init_fence();
    fence_proxy_async();
  }
  __syncthreads();
  const uint32_t ring = smem_base + plane * stages * S::STAGE;
  const uint32_t full = bars + 8 * plane * stages, empty = full + 8 * S::STAGES;
  const int row0 = (tile0 + tile) * 16;
  // this page lane's pairs of pages: pair i covers pages 2 (lanes i + plane) and the one behind it of the unit's list
  const int page_begin = u0.z * PASTA_TILE_PAGES, n_pages = min(u0.w * PASTA_TILE_PAGES, u1.z) - page_begin;
  const int32_t *pages = pv.plan + a.off_pages + u1.y + page_begin;
  const int32_t *metas = pv.plan + a.off_pmeta + u1.y + page_begin;
  const int span = ((n_pages + 1) >> 1) - plane;
  const int n_pairs = works && span > 0 ? (span + lanes - 1) / lanes : 0;
  const int n_streams = u2.x, vis_off = u2.y, tq_off = u2.z;
  const bool fin = u2.w != 0;
  const uint8_t *kv_layer = pv.kv_base + (a.layer_begin + ll) * pv.layer_stride;
  const uint16_t *scales = reinterpret_cast<const uint16_t *>(kv_layer + pv.scale_off);

  // page ids, metas and scales of 16 pairs live in registers, a page per lane; the next 16 pairs' are on their way
  auto list_index = [&](int batch) { return 2 * (lanes * (16 * batch + (lane >> 1)) + plane) + (lane & 1); };
  auto load_page = [&](int at) {
    int page = works && at < n_pages ? pages[at] : 0;
    if (page < 0 || page >= pv.n_pages) { report(pv.status, PASTA_ERR_DEVICE_CHECK); page = 0; }
    return page;
  };
  auto load_meta = [&](int at) { return works && at < n_pages ? metas[at] : -1; };     // -1: no such page
  auto load_scale = [&](int page) { return static_cast<int>(scales[static_cast<int64_t>(page) * pv.n_kv_heads + head]); };
  int cur_page = load_page(list_index(0)), nxt_page = load_page(list_index(1));
  int cur_meta = load_meta(list_index(0));
  const int64_t page_stride = static_cast<int64_t>(pv.n_kv_heads) * S::BLOCK;
  const uint8_t *kv_head = kv_layer + static_cast<int64_t>(head) * S::BLOCK;
  // brings pair i (its page ids in lanes 2 (i % 16) and the next of `page`) into stage s; lanes 0 and 1 copy a page each.
  // The page behind an odd list's last is page 0 of the pool: copied, and masked like every page that nobody sees.
  auto issue = [&](int i, int s, int page) {
    const int p = __shfl_sync(0xffffffffu, page, 2 * (i & 15) + (lane & 1));
    if (lane == 0) mbar_expect_tx(full + 8 * s, S::STAGE);
    __syncwarp();
    if (lane < 2) bulk_g2s(ring + s * S::STAGE + lane * S::BLOCK, kv_head + p * page_stride, S::BLOCK, full + 8 * s);
  };
  int issued = 0;
  // test hook: bit 0 keeps the copies back, bit 1 all warps but the producers; those that wait for them run into their limit
  const bool held = pv.debug_hold & (producer ? 1 : 2);
  if (producer && !held)
    for (; issued < stages && issued < n_pairs; ++issued) issue(issued, issued, cur_page);
  int cur_sc = load_scale(cur_page), nxt_sc = 0, nxt_meta = -1;

  // ---- the tile's query rows as fp16 A fragments: lane (g, t) holds elements [t D / 4, (t + 1) D / 4) of rows g and g + 8.
  // A row is multiplied by a power of two that brings its largest magnitude to [2^7, 2^8): bf16 numbers then fit fp16
  // exactly, down to 2^-22 of the row's largest (and to within 2^-32 of it below that).
  uint32_t qf[KS][4];
  float c1[2];                                                    // scale * log2e / (the row's factor)
  bool finite[2];
  int vis_row[2], vis[2] = {0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = row0 + h * 8 + gq;
    uint4 w[KS / 2];
#pragma unroll
    for (int k = 0; k < KS / 2; ++k) w[k] = make_uint4(0, 0, 0, 0);
    if (works && row < rows) {
      const int qn = pv.plan[a.off_tq + tq_off + (row >> g_shift)];
      const uint4 *src = reinterpret_cast<const uint4 *>(
          q + ((static_cast<int64_t>(ll) * a.n_queries + qn) * pv.n_q_heads + head * G + (row & (G - 1))) * D) + tq * (KS / 2);
#pragma unroll
      for (int k = 0; k < KS / 2; ++k) w[k] = __ldg(src + k);
    }
    vis_row[h] = row < rows ? a.off_vis + vis_off + (row >> g_shift) * n_streams : -1;
    uint32_t m2 = 0;
#pragma unroll
    for (int k = 0; k < KS / 2; ++k)
      m2 = __vmaxu2(__vmaxu2(m2, w[k].x & 0x7fff7fffu), __vmaxu2(__vmaxu2(w[k].y & 0x7fff7fffu, w[k].z & 0x7fff7fffu), w[k].w & 0x7fff7fffu));
    int amax = static_cast<int>(max(m2 >> 16, m2 & 0xffffu));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const int up = max(-126, min(126, 7 - ((amax >> 7) - 127)));
    const float f = pow2f(up);
#pragma unroll
    for (int k = 0; k < KS / 2; ++k) {                            // four elements per k-step: a word of K's codes
      qf[2 * k][h] = pack_f16(bf16_lo(w[k].x) * f, bf16_hi(w[k].x) * f);
      qf[2 * k][2 + h] = pack_f16(bf16_lo(w[k].y) * f, bf16_hi(w[k].y) * f);
      qf[2 * k + 1][h] = pack_f16(bf16_lo(w[k].z) * f, bf16_hi(w[k].z) * f);
      qf[2 * k + 1][2 + h] = pack_f16(bf16_lo(w[k].w) * f, bf16_hi(w[k].w) * f);
    }
    c1[h] = a.scale_log2 * pow2f(-up);
    finite[h] = amax < 0x7f80;
  }

  float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
  const float cap = pv.softcap_log2, cap_inv = kCap ? 1.f / cap : 0.f;
  int cur_stream = -1;
  bool ok = true;
  // this lane's addresses inside a block: K rows of its tokens (tile 1 is two rows further than tile 0), V row of the ldmatrix
  const int tok = 4 * (gq >> 1) + (gq & 1), vrow = lane & 15;

  // One pair of pages: the scores of both, one look at the reference, the products with V.  thr: per page and row half, how
  // many of the page's tokens the row sees (only looked at when kMasked).
  auto work = [&](auto masked, uint32_t blk, const int (&sc2)[2], const int (&thr)[2][2]) {
    constexpr bool kMasked = decltype(masked)::value;
    float sc[2][2][4];                                            // page, tile of 8 columns, accumulators
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        uint4 kk[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) kk[j] = lds128(blk + pg * S::BLOCK + kv8_chunk_offset<D>(0, tok + 2 * j, tq));
        const uint32_t kw[2][4] = {{kk[0].x, kk[0].y, kk[0].z, kk[0].w}, {kk[1].x, kk[1].y, kk[1].z, kk[1].w}};
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t b0, b1;
            e4m3x4_to_f16x4(kw[j][w], b0, b1);
            if (h == 0 && w == 0) mma_f16_first(sc[pg][j], qf[0], b0, b1);
            else mma_f16(sc[pg][j], qf[h * 4 + w], b0, b1);
          }
      }
    }
    // exponents: scaled, capped, masked, the V scale folded in
    bool need = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float mx = -INFINITY;
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const float c = code_factor(c1[h], static_cast<int8_t>(sc2[pg] & 0xff)), fev = static_cast<float>(static_cast<int8_t>(sc2[pg] >> 8));
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float &x = sc[pg][j][2 * h + e];
            if (kCap) x = softcap(x * capped_factor(c, cap_inv), cap) + fev;
            else x = fmaf(x, c, fev);
            if (kMasked && 4 * tq + 2 * j + e >= thr[pg][h]) x = -INFINITY;
            mx = fmaxf(mx, x);
          }
      }
      need = need || mx > ref[h] + 8.f;
    }
    if (__any_sync(0xffffffffu, need)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float mx = -INFINITY;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
          for (int j = 0; j < 2; ++j) mx = fmaxf(mx, fmaxf(sc[pg][j][2 * h], sc[pg][j][2 * h + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (mx > ref[h] + 8.f) {                                  // the same answer for the row's four lanes
          const float f = fast_exp2(ref[h] - mx);                 // 0 the first time
          ref[h] = mx;
          l[h] *= f;
#pragma unroll
          for (int n = 0; n < NT; ++n) { o[n][2 * h] *= f; o[n][2 * h + 1] *= f; }
        }
      }
    }
    uint32_t pa[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float rf = ref[h] == -INFINITY ? 0.f : ref[h];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const float p0 = fast_exp2(sc[pg][0][2 * h] - rf), p1 = fast_exp2(sc[pg][0][2 * h + 1] - rf);
        const float p2 = fast_exp2(sc[pg][1][2 * h] - rf), p3 = fast_exp2(sc[pg][1][2 * h + 1] - rf);
        l[h] = fmaf((p0 + p1) + (p2 + p3), pow2f(-static_cast<int8_t>(sc2[pg] >> 8)), l[h]);
        // fp16 weights: off by at most 2^-11 of the weight, or 2^-25 of the row's reference; the sum l keeps all bits
        pa[pg][h] = pack_f16(p0, p1);
        pa[pg][2 + h] = pack_f16(p2, p3);
      }
    }
#pragma unroll
    for (int pg = 0; pg < 2; ++pg)
#pragma unroll
      for (int c = 0; c < D / 16; c += 2) {
        uint32_t v[4];
        ldmatrix_t8(blk + pg * S::BLOCK + kv8_chunk_offset<D>(1, vrow, c + (lane >> 4)), v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t b0, b1;
          e4m3x4_to_f16x4(v[k], b0, b1);
          mma_f16(o[2 * c + k], pa[pg], b0, b1);
        }
      }
  };

  int s = 0, parity = 0;                                          // stage of pair i, and its phase
  int rs = 0, rparity = 0;                                        // stage refilled next, and the phase of its release
  for (int i = 0; i < n_pairs && (producer || !held); ++i) {
    if (i > 0 && (i & 15) == 0) {
      cur_page = nxt_page; cur_sc = nxt_sc; cur_meta = nxt_meta;
      nxt_page = load_page(list_index((i >> 4) + 1));
    }
    if ((i & 15) == 8) {                                          // by now the next page ids have arrived
      nxt_sc = load_scale(nxt_page);
      nxt_meta = load_meta(list_index((i >> 4) + 1));
    }
    const int at = 2 * (i & 15);
    const int sc2[2] = {__shfl_sync(0xffffffffu, cur_sc, at), __shfl_sync(0xffffffffu, cur_sc, at + 1)};
    const int meta[2] = {__shfl_sync(0xffffffffu, cur_meta, at), __shfl_sync(0xffffffffu, cur_meta, at + 1)};
    if (!__all_sync(0xffffffffu, mbar_wait_bounded(full + 8 * s, parity, pv.wait_limit))) { ok = false; break; }
    const uint32_t blk = ring + s * S::STAGE;
    int thr[2][2] = {{PASTA_PAGE, PASTA_PAGE}, {PASTA_PAGE, PASTA_PAGE}};
    if ((meta[0] | meta[1]) >= 0 && (meta[0] & meta[1] & PASTA_PMETA_ALL_VISIBLE)) {
      work(std::false_type(), blk, sc2, thr);
    } else {
      bool any = false;
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) {
        const int stream = meta[pg] < 0 ? cur_stream : PASTA_PMETA_STREAM(meta[pg]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (stream != cur_stream) vis[h] = vis_row[h] >= 0 ? pv.plan[vis_row[h] + stream] : 0;
          thr[pg][h] = meta[pg] < 0 ? 0 : vis[h] - PASTA_PMETA_PAGE(meta[pg]) * PASTA_PAGE;
          any = any || thr[pg][h] > 0;
        }
        cur_stream = stream;
      }
      if (__any_sync(0xffffffffu, any)) work(std::true_type(), blk, sc2, thr);
    }
    __syncwarp();                                                 // every lane is done with the stage
    if (!shared_ring) {
      if (issued < n_pairs) { issue(issued, s, issued >> 4 == i >> 4 ? cur_page : nxt_page); ++issued; }
    } else {
      if (lane == 0) mbar_arrive(empty + 8 * s);
      if (producer && i >= E_LAG && issued < n_pairs) {           // the stage of pair i - E_LAG, once everybody has left it
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(empty + 8 * rs, rparity, pv.wait_limit))) { ok = false; break; }
        issue(issued, rs, issued >> 4 == i >> 4 ? cur_page : nxt_page);
        ++issued;
        if (++rs == stages) { rs = 0; rparity ^= 1; }
      }
    }
    if (++s == stages) { s = 0; parity ^= 1; }
  }
  if (!ok) {
    // give up: report, and let the producer wait (bounded) for its copies; the outputs of this launch are undefined
    if (lane == 0) report(pv.status, PASTA_ERR_TIMEOUT);
  }
  const bool gave_up = __syncthreads_or(!ok);
  if (gave_up) {
    if (producer && works)
      for (int j = max(0, issued - stages); j < issued; ++j) mbar_wait_bounded(full + 8 * (j % stages), (j / stages) & 1);
    __syncthreads();
  }

  // ---- join the page lanes of each tile: (ref, l) and O through shared memory, where the rings were
  float *o_s = reinterpret_cast<float *>(smem + warp * S::O_BYTES);
  if (works) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = h * 8 + gq;
      float lt = l[h];
      lt += __shfl_xor_sync(0xffffffffu, lt, 1);
      lt += __shfl_xor_sync(0xffffffffu, lt, 2);
      if (tq == 0) ml_s[warp * 16 + r] = make_float2(ref[h], finite[h] ? lt : NAN);
      // 8-byte pieces: piece x of a row goes to x ^ (4 (r % 4)) so that the rows a warp writes at once spread over the banks
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *reinterpret_cast<float2 *>(o_s + r * D + (((n * 4 + tq) ^ ((r & 3) << 2)) << 1)) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
    }
  }
  __syncthreads();
  const int live = min(rows - tile0 * 16, tiles * 16);
  constexpr int PER = D / 4;                                      // threads per row, 4 elements each
  for (int x = tid; x < live * PER; x += 32 * W) {
    const int rr = x / PER, d4 = x % PER, t = rr >> 4, r = rr & 15;
    float m_all = -INFINITY;
    for (int p = 0; p < lanes; ++p) m_all = fmaxf(m_all, ml_s[(p * tiles + t) * 16 + r].x);
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l_all = 0.f, l_plain = 0.f;
    for (int p = 0; p < lanes; ++p) {
      const int w = p * tiles + t;
      const float2 ml = ml_s[w * 16 + r];
      l_plain += ml.y;
      if (ml.x == -INFINITY) continue;                            // that warp saw nothing of this row
      const float f = fast_exp2(ml.x - m_all);
      const float4 v = *reinterpret_cast<const float4 *>(smem + w * S::O_BYTES + (r * D + (((d4 * 2) ^ ((r & 3) << 2)) << 1)) * 4);
      l_all = fmaf(f, ml.y, l_all);
      acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]);
      acc[2] = fmaf(f, v.z, acc[2]); acc[3] = fmaf(f, v.w, acc[3]);
    }
    if (l_plain != l_plain) {
      m_all = not_a_row().x;
      l_all = not_a_row().y;
      acc[0] = acc[1] = acc[2] = acc[3] = NAN;
    }
    const int row = tile0 * 16 + rr;
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

template <int W, bool kCap>
cudaError_t launch_t(const PoolView &pv, const PlanHeader &h, Kv8Args a, int32_t layer_count, const void *q, cudaStream_t st) {
  using S = Kv8Smem<W>;
  static uint64_t prepared = 0;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void *>(attn_kv8_kernel<W, kCap>), S::TOTAL, &prepared);
  if (e != cudaSuccess) return e;
  a.groups = kv8_max_groups<W>((h.w[PH_T_MAX_ROWS] + 15) / 16);
  return launch_overlapped(attn_kv8_kernel<W, kCap>, dim3(h.w[PH_N_TUNITS] * a.groups, layer_count), dim3(32 * W), S::TOTAL, st,
                           pv, a, static_cast<const __nv_bfloat16 *>(q));
}

}  // namespace

cudaError_t launch_attn_kv8(const PoolView &pv, const PlanHeader &h, int32_t layer_begin, int32_t layer_count,
                            const void *q, float scale_log2, void *out, float *lse, bool out_bf16, cudaStream_t st) {
  if (pv.head_dim != D) return cudaErrorInvalidValue;
  if (h.w[PH_N_TUNITS] == 0 || layer_count == 0) return cudaSuccess;
  const Kv8Args a{h.w[PH_OFF_TUNIT], h.w[PH_OFF_PAGES], h.w[PH_OFF_PMETA], h.w[PH_OFF_VIS], h.w[PH_OFF_TQ],
                  h.w[PH_N_QUERIES], layer_begin, 1, scale_log2, out, lse, out_bf16 ? 1 : 0};
  const bool cap = pv.softcap_log2 > 0.f;
  const bool wide = h.w[PH_WHOLE_RUNS] != 0;
#define PASTA_E(WW, CC) \
  if (wide == (WW == 6) && cap == CC) return launch_t<WW, CC>(pv, h, a, layer_count, q, st);
  PASTA_E(2, false) PASTA_E(2, true) PASTA_E(6, false) PASTA_E(6, true)
#undef PASTA_E
  return cudaErrorInvalidValue;
}

}  // namespace pasta
