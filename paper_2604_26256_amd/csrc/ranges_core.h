// Equal ranges of a batch's work for the wavefronts of the stream-K decodes.
// Included by HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dora {

__device__ __forceinline__ int wave_inclusive_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(v, off);
    if (lane >= off) v += y;
  }
  return v;
}

// Number of wavefronts that take part: at most the launched count, and few
// enough that every range holds at least min_range (>= 1) page-heads, so no
// range is empty (W <= T).
__device__ __forceinline__ int effective_waves(int T, int launched, int min_range) {
  const int want = (T + min_range - 1) / min_range;
  return want < launched ? (want > 0 ? want : 1) : launched;
}

// Equal split of T page-heads into W ranges: with q = T / W and rem = T % W,
// ranges 0 .. rem-1 hold q + 1 page-heads and the others q (q >= 1).
struct Split {
  int q, rem;
  __device__ int begin(int w) const { return w * q + (w < rem ? w : rem); }
  // the range that holds page-head x
  __device__ int range_of(int x) const {
    const int big = rem * (q + 1);
    return x < big ? x / (q + 1) : rem + (x - big) / q;
  }
};

}  // namespace dora
