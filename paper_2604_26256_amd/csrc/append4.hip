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
// One wave per (sequence, page it touches, K or V, KV head).  24 runs of 300 to 700 tokens, 8 KV heads of 128
// (64 MB moved either way): stored in 17 to 20 us, read back in 18, 3.2 to 3.7 TB/s where a copy reaches
// 5; the rest is the start's chain (length, page id, rows or tiles).  A wave's codes are made eight
// tokens at a time so that its stores are words of a row: the first form, a token and a byte at a time,
// took 84 us for both.  64 x 8 tokens: 6 and 4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "decode_core.h"
#include "fp4_core.h"
#include "fp8_core.h"
#include "pages_internal.h"
#include "path_core.h"

namespace dora {

constexpr int kAppend4Waves = 8;  // of a workgroup, at most: one for each KV head

// The larger of two magnitudes, as bits: of two packed bf16 values.
__device__ __forceinline__ uint32_t top_of(uint32_t w, uint32_t top) {
  const uint32_t a = w & 0x7FFFu, c = (w >> 16) & 0x7FFFu;
  top = top > a ? top : a;
  return top > c ? top : c;
}

// Byte K of a word of codes: those of a / scale (a power of two) and b / scale.
template <int K>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, a, b, scale, K);
}

// K of a page's tokens and one head: 8 dims a lane, 64 / (D / 8) tokens at a time, the loads of four such rounds
// together.
template <int D, int P>
__device__ __forceinline__ void append4_keys(const PathParams& p, const PathPage& pg, const int* s_row,
                                             int b, int g) {
  constexpr int LANES = D / 8, AT_ONCE = 64 / LANES, CODES = P * D / 2, BATCH = 4;
  const int lane = threadIdx.x & 63, sub = lane / LANES, dim = (lane % LANES) * 8;
  const int chunk = dim >> 5;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  uint8_t* tile = p.k_pages + (pg.id * p.num_kv_heads + g) * (int64_t)Fp4<D, P>::TILE;
  const uint16_t* src = p.k_new + (int64_t)b * p.num_tokens * n + (int64_t)g * D + dim;
  const int nt = pg.hi - pg.lo;
  for (int i0 = sub; i0 - sub < nt; i0 += BATCH * AT_ONCE) {  // uniform
    u32x4 w[BATCH];
#pragma unroll
    for (int r = 0; r < BATCH; ++r) {
      const int i = i0 + r * AT_ONCE;
      w[r] = *(const u32x4*)(src + (int64_t)s_row[i < nt ? i : nt - 1] * n);
    }
#pragma unroll
    for (int r = 0; r < BATCH; ++r) {
      const int i = i0 + r * AT_ONCE;
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = top_of(w[r][k], top);
      uint32_t y = (uint32_t)__shfl_xor((int)top, 1);
      top = top > y ? top : y;
      y = (uint32_t)__shfl_xor((int)top, 2);
      top = top > y ? top : y;
      int e = (int)((top + 0x20u) >> 7) - 2;
      e = e < 1 ? 1 : e > 252 ? 252 : e;
      const bool nan = top > 0x7F80u;
      const float scale = __uint_as_float((uint32_t)e << 23);
      uint32_t codes = fp4_pair<0>(0, __uint_as_float(w[r][0] << 16), __uint_as_float(w[r][0] & 0xFFFF0000u), scale);
      codes = fp4_pair<1>(codes, __uint_as_float(w[r][1] << 16), __uint_as_float(w[r][1] & 0xFFFF0000u), scale);
      codes = fp4_pair<2>(codes, __uint_as_float(w[r][2] << 16), __uint_as_float(w[r][2] & 0xFFFF0000u), scale);
      codes = fp4_pair<3>(codes, __uint_as_float(w[r][3] << 16), __uint_as_float(w[r][3] & 0xFFFF0000u), scale);
      if (i < nt) {
        const int slot = pg.lo + i;
        *(uint32_t*)(tile + (chunk * P + slot) * 16 + (dim & 31) / 2) = nan ? 0u : codes;
        if ((lane & 3) == 0)
          tile[CODES + chunk * P + (slot & ~15) + 4 * (slot & 3) + ((slot >> 2) & 3)] =
              (uint8_t)(nan ? 255 : e);
      }
    }
  }
}

// The largest of a lane's eight values (of tokens 0 .. 7) over the 64 / PER lanes of a half: lanes share the tokens
// out, so that lane l has that of token bit_token(l & 7).
__device__ __forceinline__ int bit_token(int l) { return 4 * (l & 1) + (l & 2) + ((l >> 2) & 1); }
template <int PER>
__device__ __forceinline__ uint32_t top_of_tokens(const uint32_t (&t)[8]) {
  const int lane = threadIdx.x & 63;
  auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  uint32_t a[4], c[2], e;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool up = lane & 1;
    a[k] = larger(up ? t[k + 4] : t[k], (uint32_t)__shfl_xor((int)(up ? t[k] : t[k + 4]), 1));
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const bool up = lane & 2;
    c[k] = larger(up ? a[k + 2] : a[k], (uint32_t)__shfl_xor((int)(up ? a[k] : a[k + 2]), 2));
  }
  e = larger(lane & 4 ? c[1] : c[0], (uint32_t)__shfl_xor((int)(lane & 4 ? c[0] : c[1]), 4));
#pragma unroll
  for (int off = 8; off < 64 / PER; off <<= 1) e = larger(e, (uint32_t)__shfl_xor((int)e, off));
  return e;
}

// x / s, near enough for its E2M1 code, which changes at 0.25, 0.75, ..., 5 only: x and s have 8 bits, so that a
// quotient is one of these numbers or differs from it by 2^-10.8 of it at least.  The product with the
// reciprocal, off by 2^-22, is rounded to 13 bits: then it is that number, or on its side of it.
__device__ __forceinline__ float code_quotient(float product) {
  return __uint_as_float((__float_as_uint(product) + 0x200u) & 0xFFFFFC00u);
}

// Eight tokens of V (slots 8 k .. 8 k + 7, values w) and one head: D / 64 dims a lane; their codes as a word of a row
// for each dim, and their scales stored, where the slots are new.
template <int D, int P>
__device__ __forceinline__ void append4_eight(const uint32_t (&w)[8], const PathPage& pg, int k, uint8_t* tile,
                                              uint32_t (&words)[D / 64]) {
  typedef Fp4<D, P> F;
  constexpr int PER = D / 64;
  const int lane = threadIdx.x & 63;
  uint32_t t[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) t[u] = top_of(w[u], 0);
  const uint32_t top = top_of_tokens<PER>(t);
  const bool nan = top > 0x7F80u;
  const __bf16 rounded = (__bf16)__fdiv_rn(__uint_as_float((top < 0x7F7Fu ? top : 0x7F7Fu) << 16), 6.0f);
  const float s = fmaxf((float)rounded, 0x1p-126f);
  const int slot = 8 * k + bit_token(lane & 7);
  if ((lane & (64 / PER - 1)) < 8 && slot >= pg.lo && slot < pg.hi)
    *(uint16_t*)(tile + F::CODES + 2 * ((lane * PER >> 6) * P + slot)) =
        nan ? (uint16_t)0x7FC0 : (uint16_t)(__float_as_uint(s) >> 16);
  const float inverse = __builtin_amdgcn_rcpf(s);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    float y[8];
    auto value = [&](int u) { return __uint_as_float(i ? w[u] & 0xFFFF0000u : w[u] << 16); };
    y[0] = code_quotient(F::template times_of<0>(value(0), inverse));  // lane bit_token(u) has token u's
    y[1] = code_quotient(F::template times_of<4>(value(1), inverse));
    y[2] = code_quotient(F::template times_of<2>(value(2), inverse));
    y[3] = code_quotient(F::template times_of<6>(value(3), inverse));
    y[4] = code_quotient(F::template times_of<1>(value(4), inverse));
    y[5] = code_quotient(F::template times_of<5>(value(5), inverse));
    y[6] = code_quotient(F::template times_of<3>(value(6), inverse));
    y[7] = code_quotient(F::template times_of<7>(value(7), inverse));
    words[i] = fp4_pair<0>(0, y[0], y[1], 1.0f);
    words[i] = fp4_pair<1>(words[i], y[2], y[3], 1.0f);
    words[i] = fp4_pair<2>(words[i], y[4], y[5], 1.0f);
    words[i] = fp4_pair<3>(words[i], y[6], y[7], 1.0f);
  }
  if (__ballot(nan)) {  // uniform, rare: codes of a NaN block are 0
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (__shfl((int)nan, (lane & ~7) | bit_token(u))) {
#pragma unroll
        for (int i = 0; i < PER; ++i) words[i] &= ~(15u << (4 * u));
      }
  }
}

// V of a page's tokens and one head.  A page of new tokens: all loads together, whole rows stored.  Some of a page's:
// eight slots at a time, those of them that stay read before.
template <int D, int P>
__device__ __forceinline__ void append4_values(const PathParams& p, const PathPage& pg,
                                               const int* s_row, int b, int g) {
  constexpr int PER = D / 64, WORDS = P / 8;
  typedef typename std::conditional<PER == 2, uint32_t, uint16_t>::type value_t;
  const int lane = threadIdx.x & 63, dim = lane * PER;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  uint8_t* tile = p.v_pages + (pg.id * p.num_kv_heads + g) * (int64_t)Fp4<D, P>::TILE;
  const uint16_t* src = p.v_new + (int64_t)b * p.num_tokens * n + (int64_t)g * D + dim;
  if (pg.hi - pg.lo == P) {  // uniform
#pragma unroll 1
    for (int k = 0; k < WORDS; k += 2) {
      uint32_t w[2][8], rows[2][PER];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int u = 0; u < 8; ++u) w[j][u] = *(const value_t*)(src + (int64_t)s_row[8 * (k + j) + u] * n);
#pragma unroll
      for (int j = 0; j < 2; ++j) append4_eight<D, P>(w[j], pg, k + j, tile, rows[j]);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        *(u32x2*)(tile + (dim + i) * (P / 2) + 4 * k) = u32x2{rows[0][i], rows[1][i]};
    }
    return;
  }
  for (int k = pg.lo >> 3; 8 * k < pg.hi; ++k) {  // uniform
    uint32_t w[8], words[PER], old[PER], fresh = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int slot = 8 * k + u;
      const int i = slot < pg.lo ? 0 : slot < pg.hi ? slot - pg.lo : pg.hi - pg.lo - 1;
      w[u] = *(const value_t*)(src + (int64_t)s_row[i] * n);
      if (slot >= pg.lo && slot < pg.hi) fresh |= 15u << (4 * u);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) old[i] = *(const uint32_t*)(tile + (dim + i) * (P / 2) + 4 * k);
    append4_eight<D, P>(w, pg, k, tile, words);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      *(uint32_t*)(tile + (dim + i) * (P / 2) + 4 * k) = (old[i] & ~fresh) | (words[i] & fresh);
  }
}

template <int D, int P, bool SINGLE>
__global__ __launch_bounds__(64 * kAppend4Waves) void append4_kernel(PathParams p) {
  __shared__ int s_row[kPathMaxPage], s_bad;
  const int b = blockIdx.y;
  if (SINGLE && p.seq_lens[b] <= 0) return;  // nothing to append, nothing to report
  const PathPage pg = path_page(p, b, blockIdx.x);
  if (pg.id < 0) return;  // uniform
  if (!path_rows(p, pg, s_row, &s_bad)) return;
  for (int g = threadIdx.x >> 6; g < p.num_kv_heads; g += (int)blockDim.x >> 6) {
    if (blockIdx.z == 0)
      append4_keys<D, P>(p, pg, s_row, b, g);
    else
      append4_values<D, P>(p, pg, s_row, b, g);
  }
}

static dim3 head_waves(const PathParams& p) {
  return dim3(64u * (unsigned)(p.num_kv_heads < kAppend4Waves ? p.num_kv_heads : kAppend4Waves));
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
  const void* fn = p.head_dim == 128
                       ? (p.page_size == 16 ? append4_fn<128, 16>(single) : append4_fn<128, 32>(single))
                       : (p.page_size == 16 ? append4_fn<64, 16>(single) : append4_fn<64, 32>(single));
  return each_launch(p, [&](PathParams arg, dim3 grid, int) {
    grid.z = 2;
    void* args[] = {(void*)&arg};
    return hipLaunchKernel(fn, grid, head_waves(p), args, 0, s);
  });
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
      const uint32_t ex = tile[P * D / 2 + c * P + (slot & ~15) + 4 * (slot & 3) + ((slot >> 2) & 3)];
      const float scale = __uint_as_float(ex << 23);
#pragma unroll
      for (int k = 0; k < 4; ++k) *(bf16x8*)(o + 8 * k) = Fp4<D, P>::widen(w[k], scale);
    }
  }
}

// V: D / 64 dims a lane, whose rows it walks, two tokens at a time.
template <int D, int P, int DT>
struct ReadValues {
  static constexpr int PER = D / 64;
  static constexpr int ROW = DT == DORA_KV_BF16 ? 2 * P : DT == DORA_KV_FP8_E4M3 ? P : P / 2;  // bytes
  uint32_t rows[PER][ROW / 4];
  float scale[P / 16];  // 4-bit: of token `lane & 15` of each 16 slots

  __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
      for (int i = 0; i < ROW / 8; ++i) {
        const u32x2 two = *(const u32x2*)(tile + (lane * PER + k) * ROW + 8 * i);
        rows[k][2 * i] = two[0];
        rows[k][2 * i + 1] = two[1];
      }
    if constexpr (DT == DORA_KV_FP4) {
#pragma unroll
      for (int i = 0; i < P / 16; ++i)
        scale[i] = __uint_as_float(
            (uint32_t) * (const uint16_t*)(tile + P * D / 2 + 2 * ((lane * PER >> 6) * P + 16 * i + (lane & 15))) << 16);
    }
  }

  // Tokens U and U + 1 of the lane's dims, as bf16 words of a token each.
  template <int U>
  __device__ __forceinline__ void tokens(float page_scale, uint32_t (&out)[2]) const {
    uint32_t v[PER][2];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if constexpr (DT == DORA_KV_BF16) {
        v[k][0] = rows[k][U >> 1] & 0xFFFFu;
        v[k][1] = rows[k][U >> 1] >> 16;
      } else {
        float x, y;
        if constexpr (DT == DORA_KV_FP8_E4M3) {
          const auto two = __builtin_amdgcn_cvt_pk_f32_fp8((int)rows[k][U >> 2], (U & 2) != 0);
          x = two[0] * page_scale;
          y = two[1] * page_scale;
        } else {
          const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(rows[k][U >> 3], 1.0f, (U & 7) >> 1);
          x = Fp4<D, P>::template times_of<(U & 15)>(two[0], scale[U >> 4]);
          y = Fp4<D, P>::template times_of<(U & 15) + 1>(two[1], scale[U >> 4]);
        }
        v[k][0] = __builtin_bit_cast(uint16_t, (__bf16)x);
        v[k][1] = __builtin_bit_cast(uint16_t, (__bf16)y);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) out[i] = PER == 2 ? v[0][i] | v[PER - 1][i] << 16 : v[0][i];
  }
  template <int U>
  __device__ __forceinline__ void store(const PathPage& pg, float page_scale, uint16_t* dst, int64_t n) const {
    if constexpr (U < P) {
      uint32_t two[2];
      tokens<U>(page_scale, two);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (U + i >= pg.lo && U + i < pg.hi) {  // uniform
          uint16_t* o = dst + (int64_t)(pg.row + U + i - pg.lo) * n;
          if constexpr (PER == 2)
            *(uint32_t*)o = two[i];
          else
            *o = (uint16_t)two[i];
        }
      }
      store<U + 2>(pg, page_scale, dst, n);
    }
  }
};
template <int D, int P, int DT>
__device__ __forceinline__ void read_values(const PathParams& p, const PathPage& pg, float page_scale,
                                            uint16_t* out, int b, int g) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)p.num_kv_heads * D;
  ReadValues<D, P, DT> r;
  r.load(p.v_pages + (pg.id * p.num_kv_heads + g) * kv_page_bytes(DT, 1, P, D), lane);
  r.template store<0>(pg, page_scale, out + (int64_t)b * p.num_tokens * n + (int64_t)g * D + lane * (D / 64), n);
}

template <int D, int P, int DT>
__global__ __launch_bounds__(64 * kAppend4Waves) void kv_read_kernel(PathParams p, const float* k_scales,
                                                                    const float* v_scales,
                                                                    uint16_t* k_out, uint16_t* v_out) {
  __shared__ int s_first;
  const int b = blockIdx.y;
  PathPage pg = path_page(p, b, blockIdx.x);
  if (pg.id < 0) return;  // uniform
  if (threadIdx.x == 0) s_first = pg.row;  // without a path, the row of slot lo
  __syncthreads();
  pg.row = s_first;
  for (int g = threadIdx.x >> 6; g < p.num_kv_heads; g += (int)blockDim.x >> 6) {
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
  const void* fn = p.head_dim == 128
                       ? (p.page_size == 16 ? read_fn<128, 16>(kv_dtype) : read_fn<128, 32>(kv_dtype))
                       : (p.page_size == 16 ? read_fn<64, 16>(kv_dtype) : read_fn<64, 32>(kv_dtype));
  const int64_t row = (int64_t)p.num_tokens * p.num_kv_heads * p.head_dim;
  return each_launch(p, [&](PathParams arg, dim3 grid, int first) {
    grid.z = 2;
    uint16_t *ko = k_out + first * row, *vo = v_out + first * row;
    void* args[] = {(void*)&arg, (void*)&k_scales, (void*)&v_scales, (void*)&ko, (void*)&vo};
    return hipLaunchKernel(fn, grid, head_waves(p), args, 0, s);
  });
}

}  // namespace dora
