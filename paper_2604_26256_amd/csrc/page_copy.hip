// Whole-page copies inside one pool: forks (a sequence's last, partly filled page gets
// a copy of its own) and compaction (live pages move to free places).  Pages move as
// raw bytes, with their fp8 scales.
//
// A streaming copy bound by HBM, one workgroup per 8 KiB chunk of a page's K or V, as
// pack and unpack.  Forks copy one page many times: the loads are plain, so the
// repeats come out of the caches.  6,000 pages of 2 x 16 KiB: 393 MB in 66 us, 5.9 TB/s
// (256 pages of 2 x 32 KiB, each copied 16 times: 6 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"

namespace dora {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 2;
constexpr int kMoveBytes = kMoveThreads * kMoveUnroll * 16;  // 8 KiB
constexpr int kMoveGridPages = 32768;                        // pages per grid layer, at most

__host__ __device__ inline int move_chunks(const CopyParams& p) {
  return (int)((p.page_bytes + kMoveBytes - 1) / kMoveBytes);
}

// grid.x = K's chunks of a page, then V's; (y, z) = the page.
__global__ __launch_bounds__(kMoveThreads) void page_copy_kernel(CopyParams p) {
  const int cpp = move_chunks(p);
  const int which = (int)blockIdx.x >= cpp ? 1 : 0;  // 0: K, 1: V
  const int c = (int)blockIdx.x - which * cpp;
  const int64_t j = (int64_t)blockIdx.z * p.layer + blockIdx.y;
  if (j >= p.n_pages) return;
  const int32_t src = p.src[j], dst = p.dst[j];
  if (src < 0 || src >= p.num_pages || dst < 0 || dst >= p.num_pages) {  // skipped, reported
    if (p.dev_status && blockIdx.x == 0 && threadIdx.x == 0)
      *p.dev_status = (int32_t)DORA_ERR_DEVICE_CHECK;
    return;
  }
  if (src == dst) return;
  if (p.has_scales && c == 0 && threadIdx.x == 0) {
    float* scales = which ? p.v_scales : p.k_scales;
    scales[dst] = scales[src];
  }
  uint8_t* pages = which ? p.v_pages : p.k_pages;
  const int64_t off = (int64_t)c * kMoveBytes;
  const int64_t bytes = p.page_bytes - off < kMoveBytes ? p.page_bytes - off : kMoveBytes;
  const uint8_t* from = pages + (int64_t)src * p.page_bytes + off;
  uint8_t* to = pages + (int64_t)dst * p.page_bytes + off;
  u32x4 r[kMoveUnroll];
#pragma unroll
  for (int i = 0; i < kMoveUnroll; ++i) {
    const int64_t o = ((int64_t)i * kMoveThreads + threadIdx.x) * 16;
    if (o < bytes) r[i] = *(const u32x4*)(from + o);
  }
#pragma unroll
  for (int i = 0; i < kMoveUnroll; ++i) {
    const int64_t o = ((int64_t)i * kMoveThreads + threadIdx.x) * 16;
    if (o < bytes) __builtin_nontemporal_store(r[i], (u32x4*)(to + o));
  }
}

hipError_t launch_page_copy(const CopyParams& params, hipStream_t s) {
  CopyParams p = params;
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  if (p.n_pages <= 0) return hipSuccess;
  const int64_t z = (p.n_pages + kMoveGridPages - 1) / kMoveGridPages;
  p.layer = (int32_t)((p.n_pages + z - 1) / z);
  hipLaunchKernelGGL(page_copy_kernel,
                     dim3((unsigned)(2 * move_chunks(p)), (unsigned)p.layer, (unsigned)z),
                     dim3(kMoveThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace dora
