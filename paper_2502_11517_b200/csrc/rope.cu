// Rotary position embedding in any form (rope_form.cuh) for bf16 pools and for queries.
//
// A CTA takes a group of neighbouring tokens and a slice of the layers: it works out the tokens' sines and cosines (64 bits)
// once, into shared memory, and applies them to every head and layer of the slice.  A warp rotates 32 / (head_dim / 16) rows at
// a time, a lane one slot of 16 elements: two 16-byte loads, eight rotations, two 16-byte stores.
// What bounds it: for long prompts the instructions around the 64-bit rotation (a quarter of them are; conversions and exponents' bits
// the rest) and the latency of 16 warps per SM (three CTAs in 80 registers spill: 44 to 62 us for the queries), 50 to 60 % of what
// the bytes take; for a step the chain sine -> rotation -> store.  16384 tokens of a bf16 pool 30 us (20.5 for the bytes at the copy rate),
// 1024 query tokens of 8 layers and 32 heads 35 us (20.5), in 512 CTAs on 296 places.
#include <algorithm>

#include "device_common.cuh"
#include "kernels.hpp"
#include "page_run.cuh"
#include "rope_form.cuh"

namespace pasta {

namespace {

constexpr int R_THREADS = 256, R_WARPS = R_THREADS / 32;

__device__ __forceinline__ uint4 pack8(const float *y) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    o[i] = *reinterpret_cast<const uint32_t *>(&b);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// One slot of a bf16 row, whatever it holds: numbers that are not finite go through the same formula in fp32.
template <int D>
__device__ __forceinline__ void rotate_slot(uint4 &lo4, uint4 &hi4, const RopeForm &f, const double2 *turn, int p) {
  const bool turns = p < f.slots, alternate = f.interleaved && turns;
  if (!turns) return;
  float y[16], lo[8], hi[8];
  if (alternate) rope_slot<D>(lo4, hi4, true, turn, p, y);          // (uniform over the rotated slots: straight code for either layout)
  else rope_slot<D>(lo4, hi4, false, turn, p, y);
  if (chunk_not_finite(lo4) || chunk_not_finite(hi4)) {
    const uint32_t w[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = alternate ? bf16_lo(w[e]) : (e & 1) ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
      const float b = alternate ? bf16_hi(w[e]) : (e & 1) ? bf16_hi(w[4 + (e >> 1)]) : bf16_lo(w[4 + (e >> 1)]);
      if (fabsf(a) < INFINITY && fabsf(b) < INFINITY) continue;
      const double2 t = turn[e * (D / 16) + p];
      const float c = static_cast<float>(t.x * (1.0 / kTurnScale)), s = static_cast<float>(t.y * (1.0 / kTurnScale));
      y[e] = a * c - b * s;
      y[8 + e] = b * c + a * s;
    }
  }
  rope_unslot(y, alternate, lo, hi);
  lo4 = pack8(lo);
  hi4 = pack8(hi);
}

// the sines and cosines of tokens first .. first + cnt - 1 (pos: device array, or null for pos0 + token)
template <int D>
__device__ __forceinline__ void turns_of_group(const RopeForm &f, const int32_t *pos, int pos0, int first, int cnt, double2 *turn) {
  if (pos) {
    for (int x = threadIdx.x; x < cnt * (D / 2); x += R_THREADS)
      turn[x / (D / 2) * (D / 2) + turn_at<D>(x % (D / 2))] = turn_of(f, x % (D / 2), pos[first + x / (D / 2)]);
  } else {
    turns_of_run<D, R_THREADS>(f, pos0 + first, cnt, turn);
  }
  __syncthreads();
}

// The rows of a CTA's slice, (layer, token, head), in steps of all its warps' rows: a division per row would cost as much as a third of
// its rotation.
struct RowWalk {
  int g, r, ll, dg, dr, dl, heads, cnt;
  __device__ __forceinline__ RowWalk(int first, int step, int heads_, int cnt_) : heads(heads_), cnt(cnt_) {
    g = first % heads; r = first / heads % cnt; ll = first / (heads * cnt);
    dg = step % heads; dr = step / heads % cnt; dl = step / (heads * cnt);
  }
  __device__ __forceinline__ void next() {
    g += dg; r += dr; ll += dl;
    if (g >= heads) { g -= heads; ++r; }
    if (r >= cnt) { r -= cnt; ++ll; }
  }
};

// Where tokens go: slots in device memory (2 words per token: page, row), or the pages of a run.
struct StepSlots {
  const int32_t *slots;
  __device__ __forceinline__ int2 at(int tok) const { return make_int2(slots[2 * tok], slots[2 * tok + 1]); }
};
template <int N>
struct RunSlots {
  PageList<N> pages;
  int32_t first_offset;
  __device__ __forceinline__ int2 at(int tok) const {
    return make_int2(pages.page[(first_offset + tok) / PASTA_PAGE], (first_offset + tok) % PASTA_PAGE);
  }
};

// grid (groups of `per` tokens, slices of the layers).  A row is asked for before the row ahead of it is rotated.
template <int D, typename Slots>
__global__ void __launch_bounds__(R_THREADS, 2)
append_form_kernel(PoolView pv, const __grid_constant__ Slots slots, const int32_t *__restrict__ pos, int32_t pos0, int32_t n_tok,
                   int32_t per, int32_t layer_begin, int32_t layer_count, int32_t layers_per_cta, int64_t in_layer_stride,
                   const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new, const __grid_constant__ RopeForm form) {
  constexpr int LPT = D / 16, ROWS = 32 / LPT;
  __shared__ double2 turn[PASTA_PAGE * (D / 2)];
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, p = lane % LPT;
  const int first = blockIdx.x * per, cnt = min(per, n_tok - first), H = pv.n_kv_heads;
  const int c_a = rope_chunk_a(form, p), c_b = rope_chunk_b(form, p);
  const int ll0 = blockIdx.y * layers_per_cta, layers = min(layers_per_cta, layer_count - ll0);
  RowWalk w(warp * ROWS + lane / LPT, R_WARPS * ROWS, H, cnt);
  uint4 next[4];
  auto load = [&]() {
    const int64_t at = (ll0 + w.ll) * in_layer_stride + (static_cast<int64_t>(first + w.r) * H + w.g) * D;
    const uint4 *k = reinterpret_cast<const uint4 *>(k_new + at), *v = reinterpret_cast<const uint4 *>(v_new + at);
    next[0] = __ldg(k + c_a); next[1] = __ldg(k + c_b);
    next[2] = __ldg(v + 2 * p); next[3] = __ldg(v + 2 * p + 1);
  };
  if (w.ll < layers) load();
  turns_of_group<D>(form, pos, pos0, first, cnt, turn);
  while (w.ll < layers) {
    const int g = w.g, r = w.r, ll = ll0 + w.ll;
    uint4 ka = next[0], kb = next[1];
    const uint4 va = next[2], vb = next[3];
    w.next();
    if (w.ll < layers) load();
    const int2 slot = slots.at(first + r);
    if (slot.x < 0 || slot.x >= pv.n_pages || slot.y < 0 || slot.y >= PASTA_PAGE) {
      report(pv.status, PASTA_ERR_DEVICE_CHECK);
      continue;
    }
    rotate_slot<D>(ka, kb, form, turn + r * (D / 2), p);
    uint8_t *block = pv.kv_base + (layer_begin + ll) * pv.layer_stride + (static_cast<int64_t>(slot.x) * H + g) * kv_block_bytes(D);
    *reinterpret_cast<uint4 *>(block + kv_chunk_offset(D / 64, 0, slot.y, c_a)) = ka;
    *reinterpret_cast<uint4 *>(block + kv_chunk_offset(D / 64, 0, slot.y, c_b)) = kb;
    *reinterpret_cast<uint4 *>(block + kv_chunk_offset(D / 64, 1, slot.y, 2 * p)) = va;
    *reinterpret_cast<uint4 *>(block + kv_chunk_offset(D / 64, 1, slot.y, 2 * p + 1)) = vb;
  }
}

// q, q_out [layer_count, n, n_heads, D], possibly the same array: a lane reads its slot before it writes it, and no other lane does
template <int D>
__global__ void __launch_bounds__(R_THREADS, 2)
queries_form_kernel(const int32_t *__restrict__ pos, int32_t n, int32_t per, int32_t n_heads, int32_t layer_count, int32_t layers_per_cta,
                    const __nv_bfloat16 *q, __nv_bfloat16 *q_out, const __grid_constant__ RopeForm form) {
  constexpr int LPT = D / 16, ROWS = 32 / LPT;
  __shared__ double2 turn[PASTA_PAGE * (D / 2)];
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, p = lane % LPT;
  const int first = blockIdx.x * per, cnt = min(per, n - first);
  const int c_a = rope_chunk_a(form, p), c_b = rope_chunk_b(form, p);
  const int ll0 = blockIdx.y * layers_per_cta, layers = min(layers_per_cta, layer_count - ll0);
  RowWalk w(warp * ROWS + lane / LPT, R_WARPS * ROWS, n_heads, cnt);
  int64_t next_at = 0;
  uint4 next_a = make_uint4(0, 0, 0, 0), next_b = next_a;
  auto load = [&]() {
    next_at = ((static_cast<int64_t>(ll0 + w.ll) * n + first + w.r) * n_heads + w.g) * D;
    const uint4 *src = reinterpret_cast<const uint4 *>(q + next_at);
    next_a = src[c_a];
    next_b = src[c_b];
  };
  if (w.ll < layers) load();
  turns_of_group<D>(form, pos, 0, first, cnt, turn);
  while (w.ll < layers) {
    const int r = w.r;
    uint4 *dst = reinterpret_cast<uint4 *>(q_out + next_at);
    uint4 a = next_a, b = next_b;
    w.next();
    if (w.ll < layers) load();
    rotate_slot<D>(a, b, form, turn + r * (D / 2), p);
    dst[c_a] = a;
    dst[c_b] = b;
  }
}

// Tokens per CTA and slices of the layers.  Sharing sines and cosines (some hundred cycles each) among more rows pays only
// once every SM has two CTAs; before that, more CTAs do.
struct Split { int per, layers; };
Split split_of(int n_tok, int layer_count) {
  const int want = 148 * 2;
  const int per = std::min(PASTA_PAGE, (n_tok + want - 1) / want);
  const int groups = (n_tok + per - 1) / per;
  const int slices = std::min(layer_count, std::max(1, (want + groups - 1) / groups));
  return {per, (layer_count + slices - 1) / slices};
}

}  // namespace

namespace {

template <typename Slots>
cudaError_t launch_append(const PoolView &pv, const Slots &slots, const int32_t *pos, int32_t pos0, int32_t n_tok, int32_t layer_begin,
                          int32_t layer_count, int64_t in_layer_stride, const void *k_new, const void *v_new, const RopeForm &form,
                          cudaStream_t st) {
  const Split s = split_of(n_tok, layer_count);
  const dim3 grid((n_tok + s.per - 1) / s.per, (layer_count + s.layers - 1) / s.layers);
  const auto kernel = pv.head_dim == 128 ? append_form_kernel<128, Slots> : append_form_kernel<64, Slots>;
  kernel<<<grid, R_THREADS, 0, st>>>(pv, slots, pos, pos0, n_tok, s.per, layer_begin, layer_count, s.layers, in_layer_stride,
                                     static_cast<const __nv_bfloat16 *>(k_new), static_cast<const __nv_bfloat16 *>(v_new), form);
  return cudaGetLastError();
}

template <int N>
cudaError_t launch_append_run(const PoolView &pv, const int32_t *pages, int32_t n, int32_t first_offset, int32_t pos0, int32_t n_tok,
                              int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const void *k_new, const void *v_new,
                              const RopeForm &form, cudaStream_t st) {
  return launch_append(pv, RunSlots<N>{list_of<N>(pages, n), first_offset}, nullptr, pos0, n_tok, layer_begin, layer_count, in_layer_stride,
                       k_new, v_new, form, st);
}

}  // namespace

cudaError_t launch_kv_append_form(const PoolView &pv, const int32_t *slots, const int32_t *pos, int32_t n_tok, int32_t layer_begin,
                                  int32_t layer_count, int64_t in_layer_stride, const void *k_new, const void *v_new,
                                  const RopeForm &form, cudaStream_t st) {
  if (n_tok == 0 || layer_count == 0) return cudaSuccess;
  return launch_append(pv, StepSlots{slots}, pos, 0, n_tok, layer_begin, layer_count, in_layer_stride, k_new, v_new, form, st);
}

cudaError_t launch_kv_append_run_form(const PoolView &pv, const int32_t *pages, int32_t first_offset, int32_t pos0, int32_t n_tok,
                                      int32_t layer_begin, int32_t layer_count, int64_t in_layer_stride, const void *k_new,
                                      const void *v_new, const RopeForm &form, cudaStream_t st, int64_t *launches) {
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(k_new), *v = static_cast<const __nv_bfloat16 *>(v_new);
  const int64_t tok = static_cast<int64_t>(pv.n_kv_heads) * pv.head_dim;
  if (layer_count == 0) return cudaSuccess;
  for (int32_t done = 0; done < n_tok;) {
    const int32_t left = n_tok - done, all = (first_offset + left + PASTA_PAGE - 1) / PASTA_PAGE;
    const int32_t n = std::min(all, kPagesLarge), cnt = std::min(left, n * PASTA_PAGE - first_offset);
    const auto launch = n <= kPagesSmall ? launch_append_run<kPagesSmall> : launch_append_run<kPagesLarge>;
    const cudaError_t e = launch(pv, pages, n, first_offset, pos0 + done, cnt, layer_begin, layer_count, in_layer_stride, k + done * tok,
                                 v + done * tok, form, st);
    if (e != cudaSuccess) return e;
    *launches += 1;
    pages += n;
    done += cnt;
    first_offset = 0;
  }
  return cudaSuccess;
}

cudaError_t launch_rope_queries_form(const PoolView &pv, const int32_t *pos, int32_t n, int32_t layer_count, const void *q, void *q_out,
                                     const RopeForm &form, cudaStream_t st) {
  if (n == 0 || layer_count == 0) return cudaSuccess;
  const Split s = split_of(n, layer_count);
  const dim3 grid((n + s.per - 1) / s.per, (layer_count + s.layers - 1) / s.layers);
  const auto kernel = pv.head_dim == 128 ? queries_form_kernel<128> : queries_form_kernel<64>;
  kernel<<<grid, R_THREADS, 0, st>>>(pos, n, s.per, pv.n_q_heads, layer_count, s.layers, static_cast<const __nv_bfloat16 *>(q),
                                     static_cast<__nv_bfloat16 *>(q_out), form);
  return cudaGetLastError();
}

}  // namespace pasta
