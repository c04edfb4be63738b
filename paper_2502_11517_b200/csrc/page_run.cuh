// What the quantising stores of the 8-bit and the 4-bit cache share: the pages of a run as kernel arguments, the split of the
// layers over CTAs, and a prefetch.  Everything has internal linkage.
#pragma once
#include <algorithm>

#include "device_common.cuh"

namespace pasta {

namespace {

constexpr int A_THREADS = 256, A_WARPS = A_THREADS / 32;

// The pages of a run, as kernel arguments (a run needs no copy to the device before it); two sizes, since every launch
// carries the whole array.
template <int N> struct PageList { int32_t page[N]; };
constexpr int kPagesSmall = 64, kPagesLarge = 2048;

template <int N>
PageList<N> list_of(const int32_t *pages, int n) {
  PageList<N> list;
  std::copy(pages, pages + n, list.page);
  return list;
}

// Rows of one layer on their way into L2 while the CTA works on something else (16-byte aligned, as the loads require).
__device__ __forceinline__ void prefetch_rows(const __nv_bfloat16 *k_new, const __nv_bfloat16 *v_new, int64_t at, int bytes) {
  if (threadIdx.x < 2)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"((threadIdx.x ? v_new : k_new) + at), "r"(bytes) : "memory");
}

// layers per CTA: all layers of a page in one CTA share its sines and cosines; split only as far as the GPU has to be filled
int layers_per_cta(int groups, int layer_count) {
  const int want = 148 * 2;          // (twice as many: 35.4 against 33.3 us for 64 pages of 8 layers with rotation, 8-bit pool)
  const int slices = std::min(layer_count, std::max(1, (want + groups - 1) / groups));
  return (layer_count + slices - 1) / slices;
}

}  // namespace

}  // namespace pasta
