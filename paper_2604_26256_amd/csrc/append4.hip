// Tokens into 4-bit pages and rows back out of them (layout: fp4_core.h).
//
//   K, for each 32 dims of a token: top = the largest magnitude, as its bf16 bits
//     e = clamp(((top + 0x20) >> 7) - 2, 1, 252), codes enc(x / 2^(e - 127))
//   which is the largest's own exponent, less the codes' 2, and one more where its mantissa is
//   1.75 or above: then the largest, at most 7 steps of the lesser power, is off by no more than
//   half a step either way.
//   V, for each 64 dims: s = max(bf16(top / 6), 2^-126), codes enc(fp32(x / s))
// enc is the nearest E2M1 value, ties to the even code, +-6 where it is larger (infinities too).
// A NaN makes its block NaN: exponent 255 or a NaN scale, codes 0.  No token depends on
// another, so that several at a time are as many calls of one.
//
// One wave per (sequence, page it touches, K or V, KV head).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "decode_core.h"
#include "fp4_core.h"
#include "fp8_core.h"
#include "pages_internal.h"
#include "path_core.h"

namespace dora {

constexpr int kAppend4Waves = 4;

// The larger of two magnitudes, as bits: of two packed bf16 values.
__device__ __forceinline__ uint32_t top_of(uint32_t w, uint32_t top) {
  const uint32_t a = w & 0x7FFFu, c = (w >> 16) & 0x7FFFu;
  top = top > a ? top : a;
  return top > c ? top : c;
}

// K of one token and head: 8 dims a lane (D / 8 lanes a token), 64 / (D / 8) tokens at a time.
template <int D, int P>
__device__ __forceinline__ void append4_keys(const PathParams& p, const PathPage& pg, const int* s_row,
                                             int b, int g) {
  constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, ROUNDS = P / AT_ONCE, CODES = P * D / 2;
  const int lane = threadIdx.x & 63, sub = lane / LANES, dim = (lane % LANES) * 8;
  const int chunk = dim >> 5;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  uint8_t* tile = p.k_pages + (pg.id * p.num_kv_heads + g) * (int64_t)Fp4<D, P>::TILE;
  const uint16_t* src = p.k_new + (int64_t)b * p.num_tokens * n + (int64_t)g * D + dim;
  const int nt = pg.hi - pg.lo;
#pragma unroll 4
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = r * AT_ONCE + sub;
    if (r * AT_ONCE >= nt) break;  // uniform
    const bool mine = i < nt;
    const u32x4 w = *(const u32x4*)(src + (int64_t)s_row[mine ? i : 0] * n);
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = top_of(w[k], top);
    uint32_t y = (uint32_t)__shfl_xor((int)top, 1);
    top = top > y ? top : y;
    y = (uint32_t)__shfl_xor((int)top, 2);
    top = top > y ? top : y;
    int e = (int)((top + 0x20u) >> 7) - 2;
    e = e < 1 ? 1 : e > 252 ? 252 : e;
    const bool nan = top > 0x7F80u;
    const float scale = __uint_as_float((uint32_t)e << 23);
    uint32_t codes = 0;
#define DORA_PAIR(k)                                                                           \
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(w[k] << 16),         \
                                                   __uint_as_float(w[k] & 0xFFFF0000u), scale, k)
    DORA_PAIR(0);
    DORA_PAIR(1);
    DORA_PAIR(2);
    DORA_PAIR(3);
#undef DORA_PAIR
    if (!mine) continue;
    const int slot = pg.lo + i;
    *(uint32_t*)(tile + (chunk * P + slot) * 16 + (dim & 31) / 2) = nan ? 0u : codes;
    if ((lane & 3) == 0)
      tile[CODES + chunk * P + (slot & ~15) + 4 * (slot & 3) + ((slot >> 2) & 3)] =
          (uint8_t)(nan ? 255 : e);
  }
}

// V of a page's tokens and one head: D / 64 dims a lane, whose rows the lane puts together.
template <int D, int P>
__device__ __forceinline__ void append4_values(const PathParams& p, const PathPage& pg,
                                               const int* s_row, int b, int g) {
  constexpr int PER = D / 64, WORDS = P / 8, CODES = P * D / 2;
  const int lane = threadIdx.x & 63, dim = lane * PER;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  uint8_t* tile = p.v_pages + (pg.id * p.num_kv_heads + g) * (int64_t)Fp4<D, P>::TILE;
  const uint16_t* src = p.v_new + (int64_t)b * p.num_tokens * n + (int64_t)g * D + dim;
  uint32_t rows[PER][WORDS], old[PER][WORDS];
#pragma unroll
  for (int k = 0; k < PER; ++k)
#pragma unroll
    for (int i = 0; i < WORDS; ++i) rows[k][i] = old[k][i] = 0;
  if (pg.hi - pg.lo < P) {  // uniform: the other slots stay
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
      for (int i = 0; i < WORDS; ++i)
        old[k][i] = *(const uint32_t*)(tile + (dim + k) * (P / 2) + 4 * i);
  }
#pragma unroll
  for (int u = 0; u < P; ++u) {
    if (u < pg.lo || u >= pg.hi) continue;  // uniform
    const uint16_t* at = src + (int64_t)s_row[u - pg.lo] * n;
    const uint32_t w = PER == 2 ? *(const uint32_t*)at : (uint32_t)*at;
    uint32_t top = top_of(w, 0);
    uint32_t y;
#pragma unroll
    for (int off = 1; off < 64 / PER; off <<= 1) {
      y = (uint32_t)__shfl_xor((int)top, off);
      top = top > y ? top : y;
    }
    const bool nan = top > 0x7F80u;
    top = top < 0x7F7Fu ? top : 0x7F7Fu;
    const __bf16 rounded = (__bf16)__fdiv_rn(__uint_as_float(top << 16), 6.0f);
    const float s = fmaxf((float)rounded, 0x1p-126f);
    uint32_t codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(
        0u, __fdiv_rn(__uint_as_float(w << 16), s), __fdiv_rn(__uint_as_float(w & 0xFFFF0000u), s), 1.0f,
        0);
    if (nan) codes = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) rows[k][u >> 3] |= ((codes >> (4 * k)) & 15u) << (4 * (u & 7));
    if ((lane & (64 / PER - 1)) == 0)
      *(uint16_t*)(tile + CODES + 2 * ((dim >> 6) * P + u)) =
          nan ? (uint16_t)0x7FC0 : (uint16_t)(__float_as_uint(s) >> 16);
  }
  // slots [lo, hi) are new
  const uint64_t from = pg.lo >= 16 ? 0 : ~0ull << (4 * pg.lo), upto = pg.hi >= 16 ? ~0ull : (1ull << (4 * pg.hi)) - 1;
  const uint64_t from2 = pg.lo <= 16 ? ~0ull : ~0ull << (4 * (pg.lo - 16)),
                 upto2 = pg.hi <= 16 ? 0 : pg.hi >= 32 ? ~0ull : (1ull << (4 * (pg.hi - 16))) - 1;
#pragma unroll
  for (int k = 0; k < PER; ++k)
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const uint64_t half = i < 2 ? from & upto : from2 & upto2;
      const uint32_t fresh = (uint32_t)(half >> (32 * (i & 1)));
      *(uint32_t*)(tile + (dim + k) * (P / 2) + 4 * i) = (old[k][i] & ~fresh) | (rows[k][i] & fresh);
    }
}

template <int D, int P, bool SINGLE>
__global__ __launch_bounds__(64 * kAppend4Waves) void append4_kernel(PathParams p) {
  __shared__ int s_row[kPathMaxPage], s_bad;
  const int b = blockIdx.x;
  if (SINGLE && p.seq_lens[b] <= 0) return;  // nothing to append, nothing to report
  const PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  if (!path_rows(p, pg, s_row, &s_bad)) return;
  for (int g = threadIdx.x >> 6; g < p.num_kv_heads; g += kAppend4Waves) {
    if (blockIdx.z == 0)
      append4_keys<D, P>(p, pg, s_row, b, g);
    else
      append4_values<D, P>(p, pg, s_row, b, g);
  }
}

template <int D, int P>
static const void* append4_fn(bool single) {
  return single ? (const void*)&append4_kernel<D, P, true> : (const void*)&append4_kernel<D, P, false>;
}

hipError_t launch_append4(const PathParams& p, bool single, hipStream_t s) {
  if (p.num_seqs <= 0) return hipSuccess;
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  // pages that p.num_tokens tokens can touch
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const void* fn = p.head_dim == 128
                       ? (p.page_size == 16 ? append4_fn<128, 16>(single) : append4_fn<128, 32>(single))
                       : (p.page_size == 16 ? append4_fn<64, 16>(single) : append4_fn<64, 32>(single));
  PathParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)p.num_seqs, pages, 2), dim3(64 * kAppend4Waves), args, 0, s);
}

// ---------------------------------------------------------------------------
// read
// ---------------------------------------------------------------------------

// Rows of a page's tokens and one head, K: 16 bytes of codes or values a lane at a time.
template <int D, int P, int DT>
__device__ __forceinline__ void read_keys(const PathParams& p, const PathPage& pg, float page_scale,
                                          uint16_t* out, int b, int g) {
  constexpr int X = DT == DORA_KV_BF16 ? 8 : DT == DORA_KV_FP8_E4M3 ? 16 : 32, CHUNKS = D / X;
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  const int64_t bytes = DT == DORA_KV_FP4 ? P * D / 32 * 17 : P * D * 16 / X;
  const uint8_t* tile = p.k_pages + (pg.id * p.num_kv_heads + g) * bytes;
  uint16_t* dst = out + (int64_t)b * p.num_tokens * n + (int64_t)g * D;
  const int nt = pg.hi - pg.lo;
  for (int e = lane; e < nt * CHUNKS; e += 64) {
    const int c = e % CHUNKS, i = e / CHUNKS, slot = pg.lo + i;
    const u32x4 w = *(const u32x4*)(tile + (c * P + slot) * 16);
    uint16_t* o = dst + (int64_t)(pg.row + i) * n + c * X;
    if constexpr (DT == DORA_KV_BF16) {
      *(u32x4*)o = w;
    } else if constexpr (DT == DORA_KV_FP8_E4M3) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bf16x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[j] = (__bf16)(e4m3_to_f32((w[k] >> (8 * j)) & 0xFFu) * page_scale);
        *(bf16x4*)(o + 4 * k) = x;
      }
    } else {
      const int ex = tile[P * D / 2 + c * P + (slot & ~15) + 4 * (slot & 3) + ((slot >> 2) & 3)];
      // (a power of two that is NaN makes every value NaN, a code 0 too)
      const float scale = __uint_as_float(ex == 255 ? 0x7FC00000u : (uint32_t)ex << 23);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], 1.0f, 0),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], 1.0f, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], 1.0f, 2),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], 1.0f, 3)};
        bf16x8 x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (__bf16)((float)v[j >> 1][j & 1] * scale);
        *(bf16x8*)(o + 8 * k) = x;
      }
    }
  }
}

// V: D / 64 dims a lane, whose rows it walks.
template <int D, int P, int DT>
__device__ __forceinline__ void read_values(const PathParams& p, const PathPage& pg, float page_scale,
                                            uint16_t* out, int b, int g) {
  constexpr int PER = D / 64;
  constexpr int ROW = DT == DORA_KV_BF16 ? 2 * P : DT == DORA_KV_FP8_E4M3 ? P : P / 2;  // bytes
  const int lane = threadIdx.x & 63, dim = lane * PER;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  const int64_t bytes = DT == DORA_KV_FP4 ? P * D / 32 * 17 : D * ROW;
  const uint8_t* tile = p.v_pages + (pg.id * p.num_kv_heads + g) * bytes;
  uint16_t* dst = out + (int64_t)b * p.num_tokens * n + (int64_t)g * D + dim;
  uint32_t rows[PER][ROW / 4];
#pragma unroll
  for (int k = 0; k < PER; ++k)
#pragma unroll
    for (int i = 0; i < ROW / 4; ++i) rows[k][i] = *(const uint32_t*)(tile + (dim + k) * ROW + 4 * i);
#pragma unroll
  for (int u = 0; u < P; ++u) {
    if (u < pg.lo || u >= pg.hi) continue;  // uniform
    uint32_t two = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      uint32_t bits;
      if constexpr (DT == DORA_KV_BF16) {
        bits = (rows[k][u >> 1] >> (16 * (u & 1))) & 0xFFFFu;
      } else {
        float x;
        if constexpr (DT == DORA_KV_FP8_E4M3) {
          x = e4m3_to_f32((rows[k][u >> 2] >> (8 * (u & 3))) & 0xFFu) * page_scale;
        } else {
          const uint32_t s = *(const uint16_t*)(tile + P * D / 2 + 2 * ((dim >> 6) * P + u));
          const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(
              (rows[k][u >> 3] >> (4 * (u & 7))) & 15u, 1.0f, 0);
          x = (float)v[0] * __uint_as_float(s << 16);
        }
        bits = __builtin_bit_cast(uint16_t, (__bf16)x);
      }
      two |= bits << (16 * k);
    }
    uint16_t* o = dst + (int64_t)(pg.row + u - pg.lo) * n;
    if constexpr (PER == 2)
      *(uint32_t*)o = two;
    else
      *o = (uint16_t)two;
  }
}

template <int D, int P, int DT>
__global__ __launch_bounds__(64 * kAppend4Waves) void kv_read_kernel(PathParams p, const float* k_scales,
                                                                    const float* v_scales,
                                                                    uint16_t* k_out, uint16_t* v_out) {
  __shared__ int s_first;
  const int b = blockIdx.x;
  PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  if (threadIdx.x == 0) s_first = pg.row;  // without a path, the row of slot lo
  __syncthreads();
  pg.row = s_first;
  for (int g = threadIdx.x >> 6; g < p.num_kv_heads; g += kAppend4Waves) {
    if (blockIdx.z == 0)
      read_keys<D, P, DT>(p, pg, k_scales ? k_scales[pg.id] : 1.f, k_out, b, g);
    else
      read_values<D, P, DT>(p, pg, v_scales ? v_scales[pg.id] : 1.f, v_out, b, g);
  }
}

template <int D, int P>
static const void* read_fn(int kv_dtype) {
  return kv_dtype == DORA_KV_BF16       ? (const void*)&kv_read_kernel<D, P, DORA_KV_BF16>
         : kv_dtype == DORA_KV_FP8_E4M3 ? (const void*)&kv_read_kernel<D, P, DORA_KV_FP8_E4M3>
                                        : (const void*)&kv_read_kernel<D, P, DORA_KV_FP4>;
}

hipError_t launch_kv_read(const PathParams& p, const float* k_scales, const float* v_scales,
                          uint16_t* k_out, uint16_t* v_out, int kv_dtype, hipStream_t s) {
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const void* fn = p.head_dim == 128
                       ? (p.page_size == 16 ? read_fn<128, 16>(kv_dtype) : read_fn<128, 32>(kv_dtype))
                       : (p.page_size == 16 ? read_fn<64, 16>(kv_dtype) : read_fn<64, 32>(kv_dtype));
  PathParams arg = p;
  void* args[] = {(void*)&arg, (void*)&k_scales, (void*)&v_scales, (void*)&k_out, (void*)&v_out};
  return hipLaunchKernel(fn, dim3((unsigned)p.num_seqs, pages, 2), dim3(64 * kAppend4Waves), args, 0, s);
}

}  // namespace dora
