// Choice of the pages that a query reads: bounds of a page's keys, scores of the bounds, and
// the pages with the largest.
//
// A page's bounds, for each KV head: the largest and the smallest value of each dim over its
// tokens, as whole numbers hi[d], lo[d] in [-127, 127] times one scale
//   s = max(fp32(top / 127), 2^-126), hi = ceil(fp32(largest / s)), lo = floor(fp32(smallest / s))
// (top the largest magnitude; a NaN counts as 0, an infinity as bf16's largest number).  A query row is
// held the same way, u = rint(fp32(q / r)), r = max(fp32(top / 127), 2^-126), and its score of a page is
// what no key within the bounds exceeds:
//   max(u lo, u hi), summed over the dims  =  [max(u, 0) | min(u, 0)] . [hi | lo]
// a product of whole numbers, at most 127 * 127 * 256 < 2^24, exact in any order.  A page counts
// as the row of its KV head's group that wants it most: max over rows of fp32(r * sum), times s.  So
// the scores have no rounding that depends on the order of anything, and equal ones are equal:
// the lower page wins.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode_core.h"
#include "fp4_core.h"
#include "fp8_core.h"
#include "pages_internal.h"
#include "path_core.h"

namespace dora {

constexpr float kBf16Most = 3.3895313892515355e38f;
constexpr int kBoundsWaves = 4;

// What bounds and queries take a value for.
__device__ __forceinline__ float finite_of(float x) {
  return x == x ? fminf(fmaxf(x, -kBf16Most), kBf16Most) : 0.f;
}

// ---------------------------------------------------------------------------
// bounds
// ---------------------------------------------------------------------------

// One wave per (page, KV head).  A lane reads 16-byte pieces (a chunk of X dims of one token; 64 /
// CHUNKS tokens at a time) and keeps the extremes of its X dims; the lanes of a chunk then share
// them out, halving what each holds, until each has D / 64 dims of all tokens.
template <int D, int P, int DT>
__device__ __forceinline__ void page_bounds(const PathParams& p, const PathPage& pg, float page_scale,
                                            uint8_t* record, int g) {
  constexpr int X = DT == DORA_KV_BF16 ? 8 : DT == DORA_KV_FP8_E4M3 ? 16 : 32;
  constexpr int CHUNKS = D / X, SUBS = 64 / CHUNKS, ROUNDS = (P + SUBS - 1) / SUBS;
  const int lane = threadIdx.x & 63, chunk = lane % CHUNKS, sub = lane / CHUNKS;
  const int64_t bytes = kv_page_bytes(DT, 1, P, D);
  const uint8_t* tile = p.k_pages + (pg.id * p.num_kv_heads + g) * bytes;
  float hi[X], lo[X];
#pragma unroll
  for (int k = 0; k < X; ++k) {
    hi[k] = -__builtin_inff();
    lo[k] = __builtin_inff();
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int t = r * SUBS + sub;
    if (t >= pg.hi) continue;  // (and t >= P)
    const u32x4 w = *(const u32x4*)(tile + (chunk * P + t) * 16);
    float scale = page_scale;
    if constexpr (DT == DORA_KV_FP4) {
      const int ex = tile[P * D / 2 + chunk * P + (t & ~15) + 4 * (t & 3) + ((t >> 2) & 3)];
      scale = ex == 255 ? 0.f : __uint_as_float((uint32_t)ex << 23);  // (a NaN block counts as 0)
    }
#pragma unroll
    for (int k = 0; k < X; ++k) {
      float x;
      if constexpr (DT == DORA_KV_BF16) {
        x = __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
      } else if constexpr (DT == DORA_KV_FP8_E4M3) {
        x = e4m3_to_f32((w[k >> 2] >> (8 * (k & 3))) & 0xFFu) * scale;
      } else {
        const uint32_t two = (w[k >> 3] >> (8 * ((k >> 1) & 3))) & 0xFFu;
        const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(two, 1.0f, 0);
        x = (float)v[k & 1] * scale;
      }
      x = finite_of(x);
      hi[k] = fmaxf(hi[k], x);
      lo[k] = fminf(lo[k], x);
    }
  }
  // lanes apart by 32, 16, ..., CHUNKS: the upper one keeps the upper half of the dims
  int first = chunk * X;  // of the dims that the lane holds
  int n = X;
#pragma unroll
  for (int off = 32; off >= CHUNKS; off >>= 1) {
    const bool upper = lane & off;
    n >>= 1;
#pragma unroll
    for (int k = 0; k < X / 2; ++k) {
      if (k >= n) continue;
      const float give_hi = upper ? hi[k] : hi[k + n], give_lo = upper ? lo[k] : lo[k + n];
      hi[k] = fmaxf(upper ? hi[k + n] : hi[k], __shfl_xor(give_hi, off));
      lo[k] = fminf(upper ? lo[k + n] : lo[k], __shfl_xor(give_lo, off));
    }
    first += upper ? n : 0;
  }
  constexpr int PER = D / 64;
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) top = fmaxf(top, fmaxf(fabsf(hi[k]), fabsf(lo[k])));
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  const float s = fmaxf(__fdiv_rn(top, 127.0f), 0x1p-126f);
  uint32_t up = 0, down = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    // (top / s may round to more than 127)
    const int a = (int)fminf(fmaxf(__builtin_ceilf(__fdiv_rn(hi[k], s)), -127.f), 127.f);
    const int c = (int)fminf(fmaxf(__builtin_floorf(__fdiv_rn(lo[k], s)), -127.f), 127.f);
    up |= (uint32_t)(a & 0xFF) << (8 * k);
    down |= (uint32_t)(c & 0xFF) << (8 * k);
  }
  uint8_t* at = record + g * (2 * D) + first;
  if constexpr (PER == 2) {
    *(uint16_t*)at = (uint16_t)up;
    *(uint16_t*)(at + D) = (uint16_t)down;
  } else {
    *at = (uint8_t)up;
    at[D] = (uint8_t)down;
  }
  if (lane == 0) *(float*)(record + p.num_kv_heads * (2 * D) + 4 * g) = s;
}

template <int D, int P, int DT>
__global__ __launch_bounds__(64 * kBoundsWaves) void page_bounds_kernel(PathParams p,
                                                                       const float* k_scales,
                                                                       uint8_t* bounds) {
  const PathPage pg = path_page(p, blockIdx.x, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  const int64_t record = bounds_bytes(p.num_kv_heads, D);
  for (int g = (int)(threadIdx.x >> 6) + kBoundsWaves * (int)blockIdx.z; g < p.num_kv_heads;
       g += kBoundsWaves * (int)gridDim.z)
    page_bounds<D, P, DT>(p, pg, DT == DORA_KV_FP8_E4M3 ? k_scales[pg.id] : 1.f,
                          bounds + pg.id * record, g);
}

template <int D, int P>
static const void* bounds_fn(int kv_dtype) {
  return kv_dtype == DORA_KV_BF16       ? (const void*)&page_bounds_kernel<D, P, DORA_KV_BF16>
         : kv_dtype == DORA_KV_FP8_E4M3 ? (const void*)&page_bounds_kernel<D, P, DORA_KV_FP8_E4M3>
                                        : (const void*)&page_bounds_kernel<D, P, DORA_KV_FP4>;
}

hipError_t launch_page_bounds(const PathParams& p, const float* k_scales, uint8_t* bounds, int kv_dtype,
                              hipStream_t s) {
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const unsigned parts = (unsigned)((p.num_kv_heads + kBoundsWaves - 1) / kBoundsWaves);
  const void* fn =
      p.head_dim == 128 ? (p.page_size == 16 ? bounds_fn<128, 16>(kv_dtype) : bounds_fn<128, 32>(kv_dtype))
                        : (p.page_size == 16 ? bounds_fn<64, 16>(kv_dtype) : bounds_fn<64, 32>(kv_dtype));
  PathParams arg = p;
  void* args[] = {(void*)&arg, (void*)&k_scales, (void*)&bounds};
  return hipLaunchKernel(fn, dim3((unsigned)p.num_seqs, pages, parts), dim3(64 * kBoundsWaves), args, 0, s);
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------

constexpr int kScoreWaves = 4;
constexpr int kScoreMaxPages = 256;  // pages of a workgroup

// A query row (of the lane's column `col`, a head of the group) as whole numbers: dims 64 h + 16 grp ..
// + 15 of it for each 64 dims h, parted into max(u, 0) and min(u, 0), which meet hi and lo.
template <int D>
struct ScoreQuery {
  i32x4 up[D / 64], down[D / 64];
  float step;
};

template <int D>
__device__ __forceinline__ void score_query(ScoreQuery<D>& s, const uint16_t* qrow, bool valid) {
  const int grp = (threadIdx.x & 63) >> 4;
  u32x4 w[D / 64][2];
  float top = 0.f;
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[h][i] = valid ? *(const u32x4*)(qrow + 64 * h + 16 * grp + 8 * i) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        top = fmaxf(top, fabsf(finite_of(__uint_as_float(k & 1 ? w[h][i][k >> 1] & 0xFFFF0000u
                                                               : w[h][i][k >> 1] << 16))));
    }
  top = max_xor32(max_xor16(top));
  s.step = fmaxf(__fdiv_rn(top, 127.0f), 0x1p-126f);
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t up = 0, down = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = w[h][i >> 1][2 * (i & 1) + (k >> 1)];
        const float x = finite_of(__uint_as_float(k & 1 ? two & 0xFFFF0000u : two << 16));
        int u = (int)__builtin_rintf(__fdiv_rn(x, s.step));
        u = u > 127 ? 127 : u < -127 ? -127 : u;
        up |= (uint32_t)(u > 0 ? u : 0) << (8 * k);
        down |= (uint32_t)((u < 0 ? u : 0) & 0xFF) << (8 * k);
      }
      s.up[h][i] = (int)up;
      s.down[h][i] = (int)down;
    }
}

// Workgroup (b, part): the scores of p.chunk_pages pages of a sequence, a wave for every fourth KV head.
// Rows of a 16x16x64 product are the group's query heads, columns 16 pages: a lane reads 16 bytes of a
// page's bounds for each 64 numbers of them.
template <int D>
__global__ __launch_bounds__(64 * kScoreWaves) void page_scores_kernel(SelectParams p) {
  __shared__ int s_id[kScoreMaxPages];
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int b = blockIdx.x, first = (int)blockIdx.y * p.chunk_pages;
  const int n_seq = uni(pages_of(p.seq_lens[b], p.page_size, p.stride));
  if (first >= n_seq) return;  // uniform
  const int n = n_seq - first < p.chunk_pages ? n_seq - first : p.chunk_pages;
  for (int i = threadIdx.x; i < n; i += blockDim.x)
    s_id[i] = p.block_table[(int64_t)b * p.stride + first + i];
  __syncthreads();
  for (int g = wave; g < p.num_kv_heads; g += kScoreWaves) {
    ScoreQuery<D> q;
    score_query<D>(q, p.q + ((int64_t)b * p.num_q_heads + (int64_t)g * p.group + col) * D, col < p.group);
    float step[4];  // of the rows that the lane's results are: 4 grp + i
#pragma unroll
    for (int i = 0; i < 4; ++i) step[i] = __shfl(q.step, 4 * grp + i);
    float* out = p.scores + ((int64_t)b * p.num_kv_heads + g) * p.stride + first;
    for (int u = 0; u < n; u += 16) {
      const int i = u + col < n ? u + col : n - 1;
      const uint8_t* record = p.bounds + (int64_t)s_id[i] * p.record;
      const uint8_t* at = record + g * (2 * D) + 16 * grp;
      const float s = *(const float*)(record + p.num_kv_heads * (2 * D) + 4 * g);
      i32x4 sum{0, 0, 0, 0};
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const i32x4 hi = *(const i32x4*)(at + 64 * h), lo = *(const i32x4*)(at + D + 64 * h);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.up[h], hi, sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.down[h], lo, sum, 0, 0, 0);
      }
      float best = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * grp + k < p.group) best = fmaxf(best, (float)sum[k] * step[k]);
      best = max_xor32(max_xor16(best));
      if (grp == 0 && u + col < n) out[u + col] = best * s;
    }
  }
}

// ---------------------------------------------------------------------------
// selection
// ---------------------------------------------------------------------------

constexpr int kSelectThreads = 1024;

// Order of scores as unsigned numbers.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);  // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup per (sequence, KV head): all pages where the budget holds them; else the sinks, the most
// recent ones, and of those between the ones with the largest scores.  The score that the last
// chosen one has is found byte by byte from the top, by counts; the pages are written in order,
// those with that very score as long as there is room.
__global__ __launch_bounds__(kSelectThreads) void page_select_kernel(SelectParams p) {
  __shared__ int s_count[256];
  __shared__ int s_above, s_bin;
  __shared__ int2 s_wave[kSelectThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = blockIdx.x, b = seg / p.num_kv_heads;
  const int n = uni(pages_of(p.seq_lens[b], p.page_size, p.stride));
  int32_t* list = p.lists + (int64_t)seg * p.budget;
  if (tid == 0) p.counts[seg] = n < p.budget ? n : p.budget;
  if (n <= p.budget) {  // uniform
    for (int i = tid; i < n; i += kSelectThreads) list[i] = i;
    return;
  }
  const float* scores = p.scores + (int64_t)seg * p.stride;
  const int from = p.sinks, upto = n - p.recent;  // those that compete
  int need = p.budget - p.sinks - p.recent;       // < upto - from
  uint32_t key = 0, mask = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_count[tid] = 0;
      __syncthreads();
      for (int i = from + tid; i < upto; i += kSelectThreads) {
        const uint32_t k = score_key(scores[i]);
        if ((k & mask) == key) atomicAdd(&s_count[(k >> shift) & 255u], 1);
      }
      __syncthreads();
      if (wave == 0) {  // lane: bins 4 lane .. + 3; the first from the top whose count reaches `need`
        int c[4], mine = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          c[k] = s_count[4 * lane + k];
          mine += c[k];
        }
        int above = mine;  // in this lane's bins and those of the lanes behind
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const int y = __shfl_down(above, off);
          if (lane + off < 64) above += y;
        }
        int over = above - mine;  // in the bins behind
        if (over < need && above >= need) {
#pragma unroll
          for (int k = 3; k >= 0; --k) {
            if (over + c[k] >= need) {
              s_bin = 4 * lane + k;
              s_above = over;
              break;
            }
            over += c[k];
          }
        }
      }
      __syncthreads();
      key |= (uint32_t)s_bin << shift;
      mask |= 255u << shift;
      need -= s_above;
      __syncthreads();
    }
  }
  // `need` of those with this key are chosen, the lowest; all that have a larger one
  const bool none = p.budget == p.sinks + p.recent;
  int larger = 0, equal = 0;  // before this tile
  for (int base = 0; base < n; base += kSelectThreads) {
    const int i = base + tid;
    bool gt = false, eq = false;
    if (i < n) {
      if (i < from || i >= upto) {
        gt = true;
      } else if (!none) {
        const uint32_t k = score_key(scores[i]);
        gt = k > key;
        eq = k == key;
      }
    }
    const uint64_t gts = __ballot(gt), eqs = __ballot(eq), below = (1ull << lane) - 1;
    if (lane == 0) s_wave[wave] = make_int2(__popcll(gts), __popcll(eqs));
    __syncthreads();
    int g0 = larger, e0 = equal;
    for (int w = 0; w < kSelectThreads / 64; ++w) {
      const int2 c = s_wave[w];
      if (w < wave) {
        g0 += c.x;
        e0 += c.y;
      }
      larger += c.x;
      equal += c.y;
    }
    g0 += __popcll(gts & below);
    e0 += __popcll(eqs & below);
    if (gt || (eq && e0 < need)) list[g0 + (e0 < need ? e0 : need)] = i;
    __syncthreads();
  }
}

hipError_t launch_page_scores(const SelectParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.num_seqs, (unsigned)((p.stride + p.chunk_pages - 1) / p.chunk_pages));
  if (p.head_dim == 128)
    hipLaunchKernelGGL(page_scores_kernel<128>, grid, dim3(64 * kScoreWaves), 0, s, p);
  else
    hipLaunchKernelGGL(page_scores_kernel<64>, grid, dim3(64 * kScoreWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_page_select(const SelectParams& p, hipStream_t s) {
  hipLaunchKernelGGL(page_select_kernel, dim3((unsigned)(p.num_seqs * p.num_kv_heads)),
                     dim3(kSelectThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace dora
