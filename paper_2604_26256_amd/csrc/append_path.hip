// KV append of several tokens per sequence: the tokens of an accepted path through a
// tree of drafts, or a run of prompt tokens, go to the last positions of their
// sequence.  The pages end up as after that many single appends in order (append.hip
// has the fp8 policy), bit for bit.
//
// One workgroup per (sequence, page it touches, K or V): a page's tokens and its scale
// depend on no other page.  fp8: the scale's course over the page's tokens follows from
// the tokens' largest values alone, so these are found first.  An earlier code of the
// page goes through one requantisation for each token that makes the scale grow; the
// 256 results of all of them together are kept in a table per growth, and each code
// (an old one, or a new token's) is read, mapped and written once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "fp8_core.h"

namespace dora {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPathThreads = 256;
constexpr int kPathMaxPage = 32;  // tokens of a page, at most

// The page that workgroup (b, k) writes: its id (-1: none, or it may not be written,
// then reported), the slots [lo, hi) and the first token's place in the sequence's list.
struct PathPage {
  int64_t id;
  int lo, hi, first;
};

__device__ __forceinline__ PathPage path_page(const PathParams& p, int b, int k) {
  PathPage r{-1, 0, 0, 0};
  const int P = p.page_size, L = p.seq_lens[b];
  const int n = p.counts ? p.counts[b] : p.num_tokens;
  if (n == 0) return r;
  bool ok = n > 0 && n <= p.num_tokens && n <= L && (int64_t)L <= (int64_t)p.stride * P;
  if (ok) {
    const int base = L - n, j = base / P + k, t0 = j * P;
    if (t0 >= L) return r;  // no such page
    r.lo = base > t0 ? base - t0 : 0;
    r.hi = L - t0 < P ? L - t0 : P;
    r.first = t0 + r.lo - base;
    r.id = p.block_table[(int64_t)b * p.stride + j];
    ok = r.id >= 0 && r.id < p.num_pages;
    if (ok && p.page_owner && p.version_ids) ok = p.page_owner[r.id] == p.version_ids[b];
  }
  if (!ok) {
    if (threadIdx.x == 0 && p.dev_status) *p.dev_status = (int32_t)DORA_ERR_DEVICE_CHECK;
    r.id = -1;
  }
  return r;
}

// The source rows of the page's tokens, into s_row; false (for all threads) where one is
// no row: the page is skipped, and reported.
__device__ __forceinline__ bool path_rows(const PathParams& p, int b, const PathPage& pg, int* s_row,
                                          int* s_bad) {
  const int n = pg.hi - pg.lo;
  if (threadIdx.x == 0) *s_bad = 0;
  __syncthreads();
  if ((int)threadIdx.x < n) {
    const int i = pg.first + threadIdx.x;
    const int row = p.path ? p.path[(int64_t)b * p.num_tokens + i] : i;
    if (row < 0 || row >= p.num_tokens) *s_bad = 1;
    s_row[threadIdx.x] = row;
  }
  __syncthreads();
  if (!*s_bad) return true;
  if (threadIdx.x == 0 && p.dev_status) *p.dev_status = (int32_t)DORA_ERR_DEVICE_CHECK;
  return false;
}

// bf16.  K: a thread stores one 16-byte chunk of one token, neighbours the slots of a
// chunk.  V: a thread takes 8 head-dim rows and 8 slots, turns them round in registers
// and stores 16 bytes a row where all 8 slots are new.
__global__ __launch_bounds__(kPathThreads) void append_path_bf16_kernel(PathParams p) {
  __shared__ int s_row[kPathMaxPage], s_bad;
  const int b = blockIdx.x, P = p.page_size, n = p.num_kv_heads * p.head_dim;
  const PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  if (!path_rows(p, b, pg, s_row, &s_bad)) return;
  const int nt = pg.hi - pg.lo;
  if (blockIdx.z == 0) {
    uint8_t* page = p.k_pages + pg.id * ((int64_t)n * P * 2);
    for (int e = threadIdx.x; e < nt * (n / 8); e += kPathThreads) {
      const int c = e / nt, i = e - c * nt;
      const u32x4 x =
          *(const u32x4*)(p.k_new + ((int64_t)b * p.num_tokens + s_row[i]) * n + 8 * c);
      __builtin_nontemporal_store(x, (u32x4*)(page + ((int64_t)c * P + pg.lo + i) * 16));
    }
    return;
  }
  uint8_t* page = p.v_pages + pg.id * ((int64_t)n * P * 2);
  const int g0 = pg.lo >> 3, groups = ((pg.hi + 7) >> 3) - g0;  // groups of 8 slots
  for (int e = threadIdx.x; e < groups * (n / 8); e += kPathThreads) {
    const int c = e / groups, t0 = 8 * (g0 + e - c * groups);
    u32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + i;
      x[i] = u32x4{0u, 0u, 0u, 0u};
      if (t >= pg.lo && t < pg.hi)
        x[i] = *(const u32x4*)(p.v_new + ((int64_t)b * p.num_tokens + s_row[t - pg.lo]) * n + 8 * c);
    }
    const bool full = t0 >= pg.lo && t0 + 8 <= pg.hi;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      uint16_t* to = (uint16_t*)(page + ((int64_t)(8 * c + d) * P + t0) * 2);
      uint16_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (uint16_t)(x[i][d >> 1] >> (16 * (d & 1)));
      if (full) {
        *(u32x4*)to = u32x4{v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16,
                            v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (t0 + i >= pg.lo && t0 + i < pg.hi) to[i] = v[i];
      }
    }
  }
}

// What a page's scale does over its new tokens: scale[i] is the one token i is encoded
// with, from[i] the first growth (of `growths`) that comes after token i.
struct PathScales {
  float amax[kPathMaxPage], scale[kPathMaxPage];
  float grow_from[kPathMaxPage], grow_to[kPathMaxPage];
  int after[kPathMaxPage];
  int growths;
  float last;
};

// lut: growths x 256, row k: growths k, k + 1, ... one after the other.
template <bool IS_K>
__device__ __forceinline__ void path_side(const PathParams& p, uint8_t* pages, float* scales,
                                          const uint16_t* token) {
  __shared__ int s_row[kPathMaxPage], s_bad;
  __shared__ PathScales sc;
  __shared__ uint8_t lut[kPathMaxPage][256];
  const int b = blockIdx.x, P = p.page_size, n = p.num_kv_heads * p.head_dim, tid = threadIdx.x;
  const PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  if (!path_rows(p, b, pg, s_row, &s_bad)) return;
  const int nt = pg.hi - pg.lo;
  const uint16_t* src = token + (int64_t)b * p.num_tokens * n;
  // a wave per token: its largest magnitude
  for (int i = tid >> 6; i < nt; i += kPathThreads / 64) {
    float m = 0.f;
    const uint16_t* x = src + (int64_t)s_row[i] * n;
    for (int e = 8 * (tid & 63); e < n; e += 8 * 64) {
      const u32x4 w = *(const u32x4*)(x + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m = fmaxf(m, fabsf(bf16_bits_to_f32((uint16_t)w[k])));
        m = fmaxf(m, fabsf(bf16_bits_to_f32((uint16_t)(w[k] >> 16))));
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    if ((tid & 63) == 0) sc.amax[i] = m;
  }
  __syncthreads();
  if (tid == 0) {
    float s = pg.lo > 0 ? scales[pg.id] : 0.f;
    int growths = 0;
    for (int i = 0; i < nt; ++i) {
      const float fresh = fmaxf(__fdiv_rn(sc.amax[i], 448.0f), 0x1p-126f);
      if (pg.lo + i == 0) {
        s = fresh;
      } else if (!(fresh <= s)) {  // an unset (NaN) scale grows
        sc.grow_from[growths] = s;
        sc.grow_to[growths] = fresh;
        ++growths;
        s = fresh;
      }
      sc.scale[i] = s;
      sc.after[i] = growths;
    }
    sc.growths = growths;
    scales[pg.id] = s;
  }
  __syncthreads();
  const int growths = sc.growths;
  for (int k = growths - 1; k >= 0; --k) {
    const uint8_t c = (uint8_t)f32_to_e4m3(
        __fdiv_rn(e4m3_to_f32((uint32_t)tid) * sc.grow_from[k], sc.grow_to[k]));
    lut[k][tid] = k == growths - 1 ? c : lut[k + 1][c];
    __syncthreads();
  }
  uint8_t* page = pages + pg.id * ((int64_t)n * P);
  // Code of value x of token i after all of the page's growths.
  auto code = [&](uint16_t x, int i) {
    const uint32_t c = f32_to_e4m3(__fdiv_rn(bf16_bits_to_f32(x), sc.scale[i]));
    return sc.after[i] < growths ? (uint32_t)lut[sc.after[i]][c] : c;
  };
  if constexpr (IS_K) {
    // a thread per (16-dim chunk, slot); old slots only where they change
    const int t0 = growths ? 0 : pg.lo, per = pg.hi - t0;
    for (int e = tid; e < per * (n / 16); e += kPathThreads) {
      const int c = e / per, t = t0 + e - c * per;
      u32x4* at = (u32x4*)(page + ((int64_t)c * P + t) * 16);
      u32x4 out;
      if (t < pg.lo) {
        const u32x4 w = *at;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          out[k] = lut[0][w[k] & 0xFF] | (uint32_t)lut[0][(w[k] >> 8) & 0xFF] << 8 |
                   (uint32_t)lut[0][(w[k] >> 16) & 0xFF] << 16 | (uint32_t)lut[0][w[k] >> 24] << 24;
      } else {
        const int i = t - pg.lo;
        const u32x4* x = (const u32x4*)(src + (int64_t)s_row[i] * n + 16 * c);
        const u32x4 w0 = x[0], w1 = x[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = k < 2 ? w0[2 * k] : w1[2 * k - 4], hi = k < 2 ? w0[2 * k + 1] : w1[2 * k - 3];
          out[k] = code((uint16_t)lo, i) | code((uint16_t)(lo >> 16), i) << 8 |
                   code((uint16_t)hi, i) << 16 | code((uint16_t)(hi >> 16), i) << 24;
        }
      }
      *at = out;
    }
  } else {
    // a thread per 8 rows and 8 slots; what is not new is read, mapped and stored again
    const int g0 = growths ? 0 : pg.lo >> 3, groups = ((pg.hi + 7) >> 3) - g0;
    for (int e = tid; e < groups * (n / 8); e += kPathThreads) {
      const int c = e / groups, t0 = 8 * (g0 + e - c * groups);
      const bool full = t0 >= pg.lo && t0 + 8 <= pg.hi;
      u32x2 out[8];
#pragma unroll
      for (int d = 0; d < 8; ++d) out[d] = u32x2{0u, 0u};
      if (!full) {
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          u32x2 w = *(const u32x2*)(page + (int64_t)(8 * c + d) * P + t0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int t = t0 + i;
            uint32_t v = (w[i >> 2] >> (8 * (i & 3))) & 0xFFu;
            if (t >= pg.lo && t < pg.hi) v = 0u;
            else if (t < pg.lo && growths) v = lut[0][v];
            out[d][i >> 2] |= v << (8 * (i & 3));
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = t0 + i;
        if (t < pg.lo || t >= pg.hi) continue;
        const u32x4 x = *(const u32x4*)(src + (int64_t)s_row[t - pg.lo] * n + 8 * c);
#pragma unroll
        for (int d = 0; d < 8; ++d)
          out[d][i >> 2] |= code((uint16_t)(x[d >> 1] >> (16 * (d & 1))), t - pg.lo) << (8 * (i & 3));
      }
#pragma unroll
      for (int d = 0; d < 8; ++d) *(u32x2*)(page + (int64_t)(8 * c + d) * P + t0) = out[d];
    }
  }
}

__global__ __launch_bounds__(kPathThreads) void append_path_fp8_kernel(PathParams p) {
  if (blockIdx.z == 0)
    path_side<true>(p, p.k_pages, p.k_scales, p.k_new);
  else
    path_side<false>(p, p.v_pages, p.v_scales, p.v_new);
}

hipError_t launch_append_path(const PathParams& p, bool fp8, hipStream_t s) {
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  // pages that p.num_tokens tokens can touch
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const dim3 grid((unsigned)p.num_seqs, pages, 2);
  if (fp8)
    hipLaunchKernelGGL(append_path_fp8_kernel, grid, dim3(kPathThreads), 0, s, p);
  else
    hipLaunchKernelGGL(append_path_bf16_kernel, grid, dim3(kPathThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace dora
