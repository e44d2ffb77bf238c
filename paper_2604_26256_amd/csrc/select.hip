// Choice of the pages that a query reads: bounds of a page's keys, scores of the bounds, and
// the pages with the largest.
//
// A page's bounds, for each KV head: the largest and the smallest value of each dim over its
// tokens, as whole numbers hi[d], lo[d] in [-127, 127] times one scale
//   s = max(fp32(top / 127), 2^-126), hi = ceil(fp32(largest / s)), lo = floor(fp32(smallest / s))
// (top the largest magnitude; a NaN counts as 0, an infinity as bf16's largest number).  A query row is
// held the same way, u = rint(fp32(q / r)), r = max(fp32(top / 127), 2^-126), and its score of a page is
// what the rounded row r u gives no key within the bounds more than:
//   max(u lo, u hi), summed over the dims  =  [max(u, 0) | min(u, 0)] . [hi | lo]
// (but for 2^-24 of it where top / s rounds to more than 127, which is held to 127).  The row itself may give a
// key more, by half of r a dim: of 2,048 pages of a row 99 of 100 chosen ones are those that the
// unrounded row would choose, also where four dims of the keys, or of keys and row, are twenty times the others.
// One s for all dims of a head costs more there: 94 of 100 are those of unrounded bounds and row, but the pages
// hold as much of the softmax weight (0.43 and 0.40; 98 of 100 and 0.09 both where all dims are alike).
// a product of whole numbers, at most 127 * 127 * 256 < 2^24, exact in any order.  A page counts
// as the row of its KV head's group that wants it most: max over rows of fp32(r * sum), times s.  So
// the scores have no rounding that depends on the order of anything, and equal ones are equal:
// the lower page wins.
//
// Bounds are bound by memory and, in small calls, by their start: 1,024 rows' newest page, 8 bf16 heads (19 MB) 9.4
// us, 24 fp8 prompts of 900 to 1,900 tokens (37 MB) 11.9.  Scores: 64 long rows, 8 heads (338 MB of
// bounds) 71 us, 4.8 TB/s.  Without the products they take as long: a record of 2,080 bytes lies on
// 17 lines of 128, and no more is gained by 2 workgroups a CU, or loads past the L2 (4 spill).  Their
// choice then takes 12, a row's passes over its scores one after another.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode_core.h"
#include "fp4_core.h"
#include "fp8_core.h"
#include "pages_internal.h"
#include "path_core.h"

namespace dora {

constexpr float kBf16Most = 3.3895313892515355e38f;
constexpr int kBoundsWaves = 8;  // of a workgroup, at most: one for each KV head

// What bounds and queries take a value for.
__device__ __forceinline__ float finite_of(float x) {
  return x == x ? fminf(fmaxf(x, -kBf16Most), kBf16Most) : 0.f;
}

// ---------------------------------------------------------------------------
// bounds
// ---------------------------------------------------------------------------

typedef short s16x2 __attribute__((ext_vector_type(2)));

// bf16 numbers, two packed, as whole numbers in the same order (and back: its own inverse).
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  const s16x2 sign = __builtin_bit_cast(s16x2, w) >> 15;
  return w ^ (__builtin_bit_cast(uint32_t, sign) & 0x7FFF7FFFu);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a),
                                                                __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a),
                                                                __builtin_bit_cast(s16x2, b)));
}

// Largest of a wave's values, in every lane.
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
  return max_xor32(max_xor16(x));
}

// Lanes that hold N words each of one chunk, apart by OFF = 32, 16, ..., CHUNKS: share the words out, the
// upper lane of each pair keeping the upper half, until a lane has one.  Returns that one's place.
template <int N, int OFF, int CHUNKS, int M>
__device__ __forceinline__ int share_out(uint32_t (&hi)[M], uint32_t (&lo)[M]) {
  if constexpr (OFF < CHUNKS) {
    return 0;
  } else {
    constexpr int HALF = N > 1 ? N / 2 : 1;
    const bool upper = threadIdx.x & OFF;
#pragma unroll
    for (int k = 0; k < HALF; ++k) {
      if constexpr (N > 1) {
        const uint32_t give_hi = upper ? hi[k] : hi[k + HALF], give_lo = upper ? lo[k] : lo[k + HALF];
        hi[k] = max2(upper ? hi[k + HALF] : hi[k], (uint32_t)__shfl_xor((int)give_hi, OFF));
        lo[k] = min2(upper ? lo[k + HALF] : lo[k], (uint32_t)__shfl_xor((int)give_lo, OFF));
      } else {
        hi[k] = max2(hi[k], (uint32_t)__shfl_xor((int)hi[k], OFF));
        lo[k] = min2(lo[k], (uint32_t)__shfl_xor((int)lo[k], OFF));
      }
    }
    return (N > 1 && upper ? HALF : 0) + share_out<HALF, OFF / 2, CHUNKS>(hi, lo);
  }
}

// One wave per (page, KV head).  A lane reads 16-byte pieces (a chunk of X dims of one token; 64 /
// CHUNKS tokens at a time; behind the last token that one again) and keeps the extremes of its X dims; the
// lanes of a chunk then share them out, until each has two dims of all tokens (of 64 dims, a pair of
// lanes the same two).
//   The extremes are those of bf16 numbers, two in a word, ordered as whole numbers: fp8 and 4-bit codes
// widen to them exactly, and a page's scale keeps their order.  Where a number is odd (NaN or
// infinite, or a scale is not positive and finite) the page is looked at again, value by value.
template <int D, int P, int DT>
struct BoundsWave {
  static constexpr int X = DT == DORA_KV_BF16 ? 8 : DT == DORA_KV_FP8_E4M3 ? 16 : 32;
  static constexpr int CHUNKS = D / X, SUBS = 64 / CHUNKS, ROUNDS = (P + SUBS - 1) / SUBS;

  static __device__ __forceinline__ int exponent(const uint8_t* tile, int chunk, int t) {
    return tile[P * D / 2 + chunk * P + (t & ~15) + 4 * (t & 3) + ((t >> 2) & 3)];
  }

  // Value by value: of the dims 2 lane and 2 lane + 1 (of 64 dims, a second time in the upper lanes).
  static __device__ __forceinline__ int extremes_of_any(const uint8_t* tile, int tokens, float page_scale,
                                                        float (&hi)[2], float (&lo)[2]) {
    const int dim = 2 * ((threadIdx.x & 63) % (D / 2)), chunk = dim / X, in = dim % X;
    hi[0] = hi[1] = -__builtin_inff();
    lo[0] = lo[1] = __builtin_inff();
    for (int t = 0; t < tokens; ++t) {
      const uint8_t* at = tile + (chunk * P + t) * 16;
      float x[2];
      if constexpr (DT == DORA_KV_BF16) {
        const uint32_t two = *(const uint32_t*)(at + 2 * in);
        x[0] = __uint_as_float(two << 16);
        x[1] = __uint_as_float(two & 0xFFFF0000u);
      } else if constexpr (DT == DORA_KV_FP8_E4M3) {
        x[0] = e4m3_to_f32(at[in]) * page_scale;
        x[1] = e4m3_to_f32(at[in + 1]) * page_scale;
      } else {
        const int ex = exponent(tile, chunk, t);
        const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)at[in / 2], 1.0f, 0);
        const float scale = ex == 255 ? 0.f : __uint_as_float((uint32_t)ex << 23);  // (a NaN block: 0)
        x[0] = (float)v[0] * scale;
        x[1] = (float)v[1] * scale;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        hi[k] = fmaxf(hi[k], finite_of(x[k]));
        lo[k] = fminf(lo[k], finite_of(x[k]));
      }
    }
    return dim;
  }

  static __device__ __forceinline__ void run(const uint8_t* tile, int tokens, float page_scale,
                                             uint8_t* record, float* scale_at) {
    const int lane = threadIdx.x & 63, chunk = lane % CHUNKS, sub = lane / CHUNKS;
    u32x4 w[ROUNDS];
    int ex[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int t = r * SUBS + sub < tokens ? r * SUBS + sub : tokens - 1;
      w[r] = *(const u32x4*)(tile + (chunk * P + t) * 16);
      ex[r] = DT == DORA_KV_FP4 ? exponent(tile, chunk, t) : 0;
    }
    uint32_t hi[X / 2], lo[X / 2];
#pragma unroll
    for (int k = 0; k < X / 2; ++k) {
      hi[k] = 0x80008000u;
      lo[k] = 0x7FFF7FFFu;
    }
    bool odd = DT == DORA_KV_FP8_E4M3 && !(page_scale > 0.f && page_scale < __builtin_inff());
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      auto take = [&](int k, uint32_t two) {
        two = ordered(two);
        hi[k] = max2(hi[k], two);
        lo[k] = min2(lo[k], two);
      };
      if constexpr (DT == DORA_KV_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) take(k, w[r][k]);
      } else if constexpr (DT == DORA_KV_FP8_E4M3) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          take(2 * k, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[r][k], 1.0f, false)));
          take(2 * k + 1, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[r][k], 1.0f, true)));
        }
      } else {
        odd = odd || ex[r] == 255;
        const float scale = __uint_as_float((uint32_t)ex[r] << 23);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          take(4 * k, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][k], scale, 0)));
          take(4 * k + 1, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][k], scale, 1)));
          take(4 * k + 2, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][k], scale, 2)));
          take(4 * k + 3, __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[r][k], scale, 3)));
        }
      }
    }
    int first = chunk * X + 2 * share_out<X / 2, 32, CHUNKS>(hi, lo);
    float h[2], l[2];
    const s16x2 top2 = __builtin_bit_cast(s16x2, hi[0]), low2 = __builtin_bit_cast(s16x2, lo[0]);
    odd = odd || top2[0] > 0x7F7F || top2[1] > 0x7F7F || low2[0] < -0x7F80 || low2[1] < -0x7F80;
    if (__ballot(odd)) {  // uniform
      first = extremes_of_any(tile, tokens, page_scale, h, l);
    } else {
      const uint32_t a = ordered(hi[0]), c = ordered(lo[0]);
      h[0] = __uint_as_float(a << 16);
      h[1] = __uint_as_float(a & 0xFFFF0000u);
      l[0] = __uint_as_float(c << 16);
      l[1] = __uint_as_float(c & 0xFFFF0000u);
      if constexpr (DT == DORA_KV_FP8_E4M3) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          h[k] = finite_of(h[k] * page_scale);
          l[k] = finite_of(l[k] * page_scale);
        }
      }
    }
    const float s = fmaxf(
        __fdiv_rn(wave_max(fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(l[0]), fabsf(l[1])))), 127.0f),
        0x1p-126f);
    uint32_t up = 0, down = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      // (top / s may round to more than 127)
      const int a = (int)fminf(fmaxf(__builtin_ceilf(__fdiv_rn(h[k], s)), -127.f), 127.f);
      const int c = (int)fminf(fmaxf(__builtin_floorf(__fdiv_rn(l[k], s)), -127.f), 127.f);
      up |= (uint32_t)(a & 0xFF) << (8 * k);
      down |= (uint32_t)(c & 0xFF) << (8 * k);
    }
    *(uint16_t*)(record + first) = (uint16_t)up;
    *(uint16_t*)(record + D + first) = (uint16_t)down;
    if (lane == 0) *scale_at = s;
  }
};

template <int D, int P, int DT>
__global__ __launch_bounds__(64 * kBoundsWaves) void page_bounds_kernel(PathParams p,
                                                                       const float* k_scales,
                                                                       uint8_t* bounds) {
  const PathPage pg = path_page(p, blockIdx.y, blockIdx.x);
  if (pg.id < 0) return;  // uniform
  const int64_t record = bounds_bytes(p.num_kv_heads, D);
  for (int g = threadIdx.x >> 6; g < p.num_kv_heads; g += (int)blockDim.x >> 6) {
    uint8_t* at = bounds + pg.id * record;
    BoundsWave<D, P, DT>::run(p.k_pages + (pg.id * p.num_kv_heads + g) * kv_page_bytes(DT, 1, P, D), pg.hi,
                              DT == DORA_KV_FP8_E4M3 ? k_scales[pg.id] : 1.f, at + g * (2 * D),
                              (float*)(at + p.num_kv_heads * (2 * D)) + g);
  }
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
  const int waves = p.num_kv_heads < kBoundsWaves ? p.num_kv_heads : kBoundsWaves;
  const void* fn =
      p.head_dim == 128 ? (p.page_size == 16 ? bounds_fn<128, 16>(kv_dtype) : bounds_fn<128, 32>(kv_dtype))
                        : (p.page_size == 16 ? bounds_fn<64, 16>(kv_dtype) : bounds_fn<64, 32>(kv_dtype));
  return each_launch(p, [&](PathParams arg, dim3 grid, int) {
    void* args[] = {(void*)&arg, (void*)&k_scales, (void*)&bounds};
    return hipLaunchKernel(fn, grid, dim3(64u * (unsigned)waves), args, 0, s);
  });
}

// ---------------------------------------------------------------------------
// scores
// ---------------------------------------------------------------------------

constexpr int kScoreWaves = 4;
constexpr int kScoreMaxPages = 256;  // pages whose ids are held at a time
constexpr int kScorePerCu = 3;       // workgroups of a CU

// The bounds of 16 pages for one KV head as operands of D / 32 16x16x64 products: lane (col, grp) has of page col the
// bytes D / 2 * grp + 16 m for product m.  A page's bounds lie together and pages apart, so loads in this
// order would be one line a lane (four times the time: the address unit takes 64 bytes of one line a
// cycle).  They are made with the M = D / 32 lanes of a group on neighbouring bytes of one page: load s, lane i of its group
// reads piece i of the page that operand lane s of the group wants, and the group's lanes and the
// registers are then exchanged.
template <int M>
struct PageBounds {
  i32x4 w[M];
};

// Lanes apart by OFF and registers a, b: lane bit and register change places.
template <int OFF>
__device__ __forceinline__ void exchange(i32x4& a, i32x4& b) {
  constexpr int DOWN = OFF == 1 ? 0xA0 : 0x44, UP = OFF == 1 ? 0xF5 : 0xEE;  // quad_perm: from the lower, the upper one
  const bool upper = threadIdx.x & OFF;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int from_b = __builtin_amdgcn_update_dpp(0, b[k], DOWN, 0xF, 0xF, true);
    const int from_a = __builtin_amdgcn_update_dpp(0, a[k], UP, 0xF, 0xF, true);
    a[k] = upper ? from_b : a[k];
    b[k] = upper ? b[k] : from_a;
  }
}
template <int M>
__device__ __forceinline__ void as_operands(PageBounds<M>& x) {
  if constexpr (M == 4) {
    exchange<1>(x.w[0], x.w[1]);
    exchange<1>(x.w[2], x.w[3]);
    exchange<2>(x.w[0], x.w[2]);
    exchange<2>(x.w[1], x.w[3]);
  } else {
    exchange<1>(x.w[0], x.w[1]);
  }
}

// The rows of a group's 16 columns, D / 4 values of one a lane (row lane >> 2; rows that are none are 0).
template <int D>
struct ScoreRows {
  u32x4 w[D / 32];
};
template <int D>
__device__ __forceinline__ void load_rows(ScoreRows<D>& s, const uint16_t* group_rows, int group) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
    s.w[i] = lane >> 2 < group ? *(const u32x4*)(group_rows + (lane >> 2) * D + D / 4 * (lane & 3) + 8 * i)
                               : u32x4{0u, 0u, 0u, 0u};
}

// The rows as whole numbers, into LDS: u[16][D], and their steps.
template <int D>
__device__ __forceinline__ void whole_rows(ScoreRows<D>& s, uint8_t* u, float* steps) {
  const int lane = threadIdx.x & 63;
  constexpr int N = D / 32;  // 8 values each
  u32x4(&w)[N] = s.w;
  uint32_t most = 0;  // the largest magnitudes, two
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) most = max2(most, w[i][k] & 0x7FFF7FFFu);
  most = max2(most, most >> 16) & 0xFFFFu;
  const bool odd = most > 0x7F7Fu;  // a NaN or an infinity
  if (__ballot(odd)) {              // uniform, rare: each value for what it counts
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = finite_of(__uint_as_float(w[i][k] << 16));
        const float y = finite_of(__uint_as_float(w[i][k] & 0xFFFF0000u));
        w[i][k] = (__float_as_uint(x) >> 16) | (__float_as_uint(y) & 0xFFFF0000u);
        top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
      }
    most = __float_as_uint(top) >> 16;
  }
  float top = __uint_as_float(most << 16);
  top = fmaxf(top, __shfl_xor(top, 1));
  top = fmaxf(top, __shfl_xor(top, 2));
  float step = fmaxf(__fdiv_rn(top, 127.0f), 0x1p-126f);
  if ((lane & 3) == 0) steps[lane >> 2] = step;
  // fp32(x / step): the product with the rounded reciprocal, corrected once by what it leaves, is
  // the rounded quotient (Markstein, "Computation of elementary functions on the IBM RISC System/6000
  // processor", 1990), as long as what is left is not below the normal numbers
  if (__ballot(step < 0x1p-90f)) {  // uniform, rare: the same quotients 2^64 higher up, exactly
    const float up = step < 0x1p-90f ? 0x1p64f : 1.f;
    step *= up;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[i][k] = __float_as_uint(__uint_as_float(w[i][k] << 16) * up) >> 16 |
                  __float_as_uint(__uint_as_float(w[i][k] & 0xFFFF0000u) * up);
  }
  const float inverse = __fdiv_rn(1.0f, step);
  uint8_t* to = u + (lane >> 2) * D + D / 4 * (lane & 3);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x2 eight;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t four = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = w[i][2 * j + (k >> 1)];
        const float x = __uint_as_float(k & 1 ? two & 0xFFFF0000u : two << 16);
        float y = x * inverse;
        y = __builtin_fmaf(__builtin_fmaf(-y, step, x), inverse, y);
        four |= (uint32_t)((int)__builtin_rintf(y) & 0xFF) << (8 * k);  // (of at most 127.00001)
      }
      eight[j] = four;
    }
    *(u32x2*)(to + 8 * i) = eight;
  }
}

// The rows as an operand, for the bytes that a lane has of a page: max(u, 0) against the largest values, in the
// lower two lane groups, min(u, 0) against the smallest in the upper two; and the steps of the rows
// that the lane's results are.
template <int D>
struct ScoreQuery {
  i32x4 w[D / 32];
  f32x4 step;
};
template <int D>
__device__ __forceinline__ void query_operand(ScoreQuery<D>& q, const uint8_t* u, const float* steps) {
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  q.step = *(const f32x4*)(steps + 4 * grp);
#pragma unroll
  for (int m = 0; m < D / 32; ++m) {
    q.w[m] = *(const i32x4*)(u + col * D + D / 2 * (grp & 1) + 16 * m);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (uint32_t)q.w[m][i], negative = ((w >> 7) & 0x01010101u) * 0xFFu;
      q.w[m][i] = (int)(grp < 2 ? w & ~negative : w & negative);
    }
  }
}

// The largest score of a page's over the group's rows, in all lanes of its column: sum and step are of
// rows 4 * (lane >> 4) .. + 3.
__device__ __forceinline__ float best_row(i32x4 sum, f32x4 step, int group) {
  const int grp = (threadIdx.x & 63) >> 4;
  float best = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (4 * grp + k < group) best = fmaxf(best, (float)sum[k] * step[k]);
  return max_xor32(max_xor16(best));
}

// A wave's place in the batch's list of tiles (16 pages of a sequence): every workgroup takes an equal
// contiguous range, however long the sequences are.  By all threads of a workgroup; to: the range,
// and the sequence and tile that it starts with.
struct ScoreRange {
  int count, b, tile, pages;  // tiles of the range; where it starts, and the pages of that sequence
};
__device__ __forceinline__ ScoreRange score_range(const SelectParams& p) {
  constexpr int THREADS = 64 * kScoreWaves;
  __shared__ int s_wave[kScoreWaves], s_at[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = p.num_seqs;
  auto pages_at = [&](int b) { return b < B ? pages_of(p.seq_lens[b], p.page_size, p.stride) : 0; };
  const int own = pages_at(tid);
  int sum = (own + 15) / 16;
  for (int b = tid + THREADS; b < B; b += THREADS) sum += (pages_at(b) + 15) / 16;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
  if (lane == 0) s_wave[wave] = sum;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kScoreWaves; ++w) total += s_wave[w];
  const int x0 = (int)((int64_t)total * blockIdx.x / gridDim.x);
  ScoreRange r{(int)((int64_t)total * (blockIdx.x + 1) / gridDim.x) - x0, 0, 0, 0};
  if (r.count == 0) return r;  // uniform
  int before = 0;
  for (int base = 0; base < B; base += THREADS) {
    const int b = base + tid, pages = base ? pages_at(b) : own, n = (pages + 15) / 16;
    int incl = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    __syncthreads();  // (s_wave is read)
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kScoreWaves; ++w) {
      if (w < wave) incl += s_wave[w];
      all += s_wave[w];
    }
    const int last = before + incl, first = last - n;
    if (first <= x0 && x0 < last) {
      s_at[0] = b;
      s_at[1] = x0 - first;
      s_at[2] = pages;
    }
    before += all;
    if (before > x0) break;  // uniform
  }
  __syncthreads();
  r.b = uni(s_at[0]);
  r.tile = uni(s_at[1]);
  r.pages = uni(s_at[2]);
  return r;
}

// A wave takes two KV heads at a time (512 bytes of a page's bounds, one behind the other), whose query rows it holds
// as operands; the four waves have a pair of heads each or, with fewer pairs, every second or fourth tile of one.
// Rows of a 16x16x64 product are a group's query heads, columns the pages.
template <int D>
__global__ __launch_bounds__(64 * kScoreWaves, kScorePerCu) void page_scores_kernel(SelectParams p) {
  constexpr int M = D / 32;
  __shared__ int s_id[kScoreMaxPages];
  __shared__ float s_out[kScoreWaves][2][kScoreMaxPages];  // (a store each time would be waited for with later loads)
  __shared__ __align__(16) uint8_t s_u[kScoreWaves][2][16][D];
  __shared__ __align__(16) float s_step[kScoreWaves][2][16];
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int Hkv = p.num_kv_heads, pairs = (Hkv + 1) / 2;
  const int ways = pairs == 1 ? 4 : pairs == 2 ? 2 : 1;  // waves that share a pair's tiles
  ScoreRange at = score_range(p);
  int held = -1;  // the sequence and pair whose rows are in q
  ScoreQuery<D> q[2];
  auto hold_pair = [&](int pair, auto meanwhile) {
    ScoreRows<D> rows[2];
    const bool other = held != at.b * pairs + pair;  // uniform
    if (other) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // (one head: the same again)
        const int g = 2 * pair + h < Hkv ? 2 * pair + h : Hkv - 1;
        load_rows<D>(rows[h], p.q + ((int64_t)at.b * p.num_q_heads + (int64_t)g * p.group) * D, p.group);
      }
    }
    meanwhile();
    if (!other) return;
    held = at.b * pairs + pair;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h) whole_rows<D>(rows[h], s_u[wave][h][0], s_step[wave][h]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h) query_operand<D>(q[h], s_u[wave][h][0], s_step[wave][h]);
  };
  while (at.count > 0) {  // uniform
    const int n_seq = at.pages, tiles = (n_seq + 15) / 16;
    if (at.tile >= tiles) {  // the next sequence
      ++at.b;
      at.tile = 0;
      at.pages = uni(pages_of(p.seq_lens[at.b], p.page_size, p.stride));
      continue;
    }
    int n_tiles = tiles - at.tile < at.count ? tiles - at.tile : at.count;
    n_tiles = n_tiles < kScoreMaxPages / 16 ? n_tiles : kScoreMaxPages / 16;
    const int first = 16 * at.tile, n = n_seq - first < 16 * n_tiles ? n_seq - first : 16 * n_tiles;
    // the ids, and beside them the rows of the wave's first pair
    static_assert(kScoreMaxPages == 64 * kScoreWaves, "an id a thread");
    const int id = p.block_table[(int64_t)at.b * p.stride + first + ((int)threadIdx.x < n ? (int)threadIdx.x : n - 1)];
    const int pair0 = wave / ways;
    hold_pair(pair0 < pairs ? pair0 : 0, [&]() {
      __syncthreads();  // (s_id is read)
      s_id[threadIdx.x] = id;
    });
    __syncthreads();
    for (int pair = pair0; pair < pairs; pair += kScoreWaves / ways) {
      const int g0 = 2 * pair, heads = Hkv - g0 < 2 ? 1 : 2;
      if (pair != pair0) hold_pair(pair, []() {});
      // a tile's bounds; behind the last tile its loads are made again: under a branch they would be waited for
      // with those before them
      const int head2 = heads == 2 ? 2 * D : 0;  // (one head: the same again)
      struct Tile {
        PageBounds<M> x[2];
        float s;  // of head grp & 1
      };
      auto load = [&](Tile& t, int u) {
        u = u < n_tiles ? u : n_tiles - 1;
        auto page = [&](int i) {
          i += 16 * u;
          return p.bounds + (int64_t)s_id[i < n ? i : n - 1] * p.record;
        };
#pragma unroll
        for (int k = 0; k < M; ++k) {
          const uint8_t* from = page((col & ~(M - 1)) + k) + D / 2 * grp + 16 * (col & (M - 1)) + g0 * (2 * D);
          t.x[0].w[k] = *(const i32x4*)from;
          t.x[1].w[k] = *(const i32x4*)(from + head2);
        }
        t.s = ((const float*)(page(col) + Hkv * (2 * D)))[g0 + ((grp & 1) < heads ? grp & 1 : 0)];
      };
      auto score = [&](Tile& t, int u) {
        float best[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          i32x4 sum{0, 0, 0, 0};
          as_operands<M>(t.x[h]);
#pragma unroll
          for (int m = 0; m < M; ++m)
            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[h].w[m], t.x[h].w[m], sum, 0, 0, 0);
          best[h] = best_row(sum, q[h].step, p.group);
        }
        if (grp < 2) s_out[wave][grp][16 * u + col] = (grp ? best[1] : best[0]) * t.s;
      };
      Tile t[2];
      int u = wave % ways;
      load(t[0], u);
      while (u < n_tiles) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          load(t[r ^ 1], u + ways);
          score(t[r], u);
          u += ways;
          if (u >= n_tiles) break;
        }
      }
      // this wave's scores of its tiles (LDS serves a wave's accesses in order)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      float* out = p.scores + ((int64_t)at.b * Hkv + g0) * p.stride + first;
      for (int h = 0; h < heads; ++h)
        for (int i = lane; i < n; i += 64)
          if ((i >> 4) % ways == wave % ways) out[(int64_t)h * p.stride + i] = s_out[wave][h][i];
    }
    at.count -= n_tiles;
    at.tile += n_tiles;
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

// Of the n > budget pages of a segment the sinks, the most recent ones, and of those between the ones
// with the largest scores, into list: by all threads of a workgroup.  The last chosen one's score is
// found from its upper bits down, 8 at a time below those that all scores share, by counting; the
// pages are written in order, those with that very score as long as there is room.
//   ITEMS: scores that a thread holds in registers (score_at(i) of i = tid + k * kSelectThreads); 0: any
// number of them, asked for again each time.
template <int ITEMS, typename ScoreAt>
__device__ __forceinline__ void choose_pages(const SelectParams& p, int n, int32_t* list, ScoreAt score_at) {
  constexpr int WAVES = kSelectThreads / 64;
  __shared__ int s_count[256];
  __shared__ int s_above, s_bin, s_all;
  __shared__ uint32_t s_low[WAVES], s_high[WAVES];
  __shared__ int2 s_part[(ITEMS ? ITEMS : 1) * WAVES];  // {larger, equal} of a wave's 64 pages
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int from = p.sinks, upto = n - p.recent;  // those that compete
  int need = p.budget - p.sinks - p.recent;       // < upto - from
  uint32_t held[ITEMS ? ITEMS : 1];
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int i = tid + k * kSelectThreads;
      held[k] = score_key(i < n ? score_at(i) : 0.f);
    }
  }
  auto competes = [&](int i) { return i >= from && i < upto; };
  auto each = [&](auto f) {  // f(page, key) for this thread's pages that compete
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
        if (competes(tid + k * kSelectThreads)) f(tid + k * kSelectThreads, held[k]);
    } else {
      for (int i = from + tid; i < upto; i += kSelectThreads) f(i, score_key(score_at(i)));
    }
  };
  uint32_t key = 0;
  const bool some = need > 0;  // uniform
  if (some) {
    uint32_t low = ~0u, high = 0;
    each([&](int, uint32_t k) {
      low = low < k ? low : k;
      high = high > k ? high : k;
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      const uint32_t l = (uint32_t)__shfl_xor((int)low, off), h = (uint32_t)__shfl_xor((int)high, off);
      low = low < l ? low : l;
      high = high > h ? high : h;
    }
    if (lane == 0) {
      s_low[wave] = low;
      s_high[wave] = high;
    }
    if (tid < 256) s_count[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      low = low < s_low[w] ? low : s_low[w];
      high = high > s_high[w] ? high : s_high[w];
    }
    int left = low == high ? 0 : 32 - __builtin_clz(low ^ high);  // bits that are not shared
    left = uni(left);
    key = left < 32 ? high >> left : 0;  // the upper bits that are known
    while (left > 0) {
      const int take = left < 8 ? left : 8, shift = left - take;
      each([&](int, uint32_t k) {
        if ((left < 32 ? k >> left : 0) == key) atomicAdd(&s_count[(k >> shift) & ((1u << take) - 1)], 1);
      });
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
              s_all = over + c[k] == need;
              break;
            }
            over += c[k];
          }
        }
      }
      __syncthreads();
      key = key << take | (uint32_t)s_bin;
      need -= s_above;
      left = shift;
      if (s_all) {  // uniform: all scores that begin like this are chosen, whatever their lower bits
        key = (key << left) - 1;  // (at least one is not chosen: not below 0)
        need = 0;
        break;
      }
      if (left > 0) {
        if (tid < 256) s_count[tid] = 0;
        __syncthreads();
      }
    }
  }
  // `need` of those with this key are chosen, the lowest; all that have a larger one
  auto place = [&](int i, uint32_t k, bool& gt, bool& eq) {
    gt = i < n && (!competes(i) || (some && k > key));
    eq = i < n && competes(i) && some && k == key;
  };
  const uint64_t below = (1ull << lane) - 1;
  if constexpr (ITEMS > 0) {
    uint64_t gts[ITEMS], eqs[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      bool gt, eq;
      place(tid + k * kSelectThreads, held[k], gt, eq);
      gts[k] = __ballot(gt);
      eqs[k] = __ballot(eq);
      if (lane == 0) s_part[k * WAVES + wave] = make_int2(__popcll(gts[k]), __popcll(eqs[k]));
    }
    __syncthreads();
    if (wave == 0) {  // the numbers before each wave's pages
      constexpr int PER = (ITEMS * WAVES + 63) / 64;
      int2 c[PER];
      int g = 0, e = 0;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int i = lane * PER + k;
        c[k] = i < ITEMS * WAVES ? s_part[i] : make_int2(0, 0);
        g += c[k].x;
        e += c[k].y;
      }
      int gi = g, ei = e;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(gi, off), z = __shfl_up(ei, off);
        if (lane >= off) {
          gi += y;
          ei += z;
        }
      }
      g = gi - g;
      e = ei - e;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int i = lane * PER + k;
        if (i < ITEMS * WAVES) s_part[i] = make_int2(g, e);
        g += c[k].x;
        e += c[k].y;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int2 c = s_part[k * WAVES + wave];
      const int e0 = c.y + __popcll(eqs[k] & below);
      const bool gt = (gts[k] >> lane) & 1, eq = (eqs[k] >> lane) & 1;
      if (gt || (eq && e0 < need))
        list[c.x + __popcll(gts[k] & below) + (e0 < need ? e0 : need)] = tid + k * kSelectThreads;
    }
  } else {
    int larger = 0, equal = 0;  // before this round
    for (int base = 0; base < n; base += kSelectThreads) {
      const int i = base + tid;
      bool gt, eq;
      place(i, i < n ? score_key(score_at(i)) : 0u, gt, eq);
      const uint64_t gts = __ballot(gt), eqs = __ballot(eq);
      if (lane == 0) s_part[wave] = make_int2(__popcll(gts), __popcll(eqs));
      __syncthreads();
      int g0 = larger, e0 = equal;
      for (int w = 0; w < WAVES; ++w) {
        const int2 c = s_part[w];
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
}

// A segment's count, and its list where the budget holds all its pages.  False: they have to be chosen.
__device__ __forceinline__ bool lists_all(const SelectParams& p, int seg, int n, int32_t* list) {
  if (threadIdx.x == 0) p.counts[seg] = n < p.budget ? n : p.budget;
  if (n > p.budget) return false;  // uniform
  for (int i = threadIdx.x; i < n; i += kSelectThreads) list[i] = i;
  return true;
}

// One workgroup per (sequence, KV head).
template <int ITEMS>
__global__ __launch_bounds__(kSelectThreads) void page_select_kernel(SelectParams p) {
  const int seg = blockIdx.x, b = seg / p.num_kv_heads;
  const int n = uni(pages_of(p.seq_lens[b], p.page_size, p.stride));
  int32_t* list = p.lists + (int64_t)seg * p.budget;
  if (lists_all(p, seg, n, list)) return;
  const float* scores = p.scores + (int64_t)seg * p.stride;
  choose_pages<ITEMS>(p, n, list, [&](int i) { return scores[i]; });
}

// A row as whole numbers by one wave, two of them a lane (of 64 values, the upper lanes' are not stored): into
// u[D], and its step.
template <int D>
__device__ __forceinline__ void score_row(const uint16_t* qrow, bool valid, uint16_t* u, float* step_at) {
  const int lane = threadIdx.x & 63, at = lane % (D / 2);
  const uint32_t two = valid ? ((const uint32_t*)qrow)[at] : 0u;
  const float x = finite_of(__uint_as_float(two << 16)), y = finite_of(__uint_as_float(two & 0xFFFF0000u));
  const float step = fmaxf(__fdiv_rn(wave_max(fmaxf(fabsf(x), fabsf(y))), 127.0f), 0x1p-126f);
  const int a = (int)__builtin_rintf(__fdiv_rn(x, step)), b = (int)__builtin_rintf(__fdiv_rn(y, step));
  if (lane < D / 2) u[at] = (uint16_t)((a & 0xFF) | (b & 0xFF) << 8);
  if (lane == 0) *step_at = step;
}

// Scores and choice in one launch, for few and short rows: one workgroup per (sequence, KV head).  A wave
// makes one row of the group whole numbers, for all of them, and has every sixteenth tile of 16 pages.
template <int D>
__global__ __launch_bounds__(kSelectThreads) void page_score_select_kernel(SelectParams p) {
  constexpr int M = D / 32, WAVES = kSelectThreads / 64, TILES = kSelectThreads / 16 / WAVES;
  __shared__ float s_score[kSelectThreads];
  __shared__ __align__(16) float s_step[16];
  __shared__ __align__(16) uint8_t s_u[16][D];
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int Hkv = p.num_kv_heads, seg = blockIdx.x, b = seg / Hkv, g = seg - b * Hkv;
  int id[TILES];  // of page `col` of each tile (loaded beside the length)
#pragma unroll
  for (int k = 0; k < TILES; ++k) {
    const int i = 16 * (wave + k * WAVES) + col;
    id[k] = p.block_table[(int64_t)b * p.stride + (i < p.stride ? i : p.stride - 1)];
  }
  const int n = uni(pages_of(p.seq_lens[b], p.page_size, p.stride));
  int32_t* list = p.lists + (int64_t)seg * p.budget;
  const bool all = lists_all(p, seg, n, list);
  if (all && !p.scores) return;  // uniform
  score_row<D>(p.q + ((int64_t)b * p.num_q_heads + (int64_t)g * p.group + wave) * D, wave < p.group,
               (uint16_t*)s_u[wave], &s_step[wave]);
  const int mine = 16 * wave < n ? (((n + 15) >> 4) - wave + WAVES - 1) / WAVES : 0;  // tiles
  PageBounds<M> x[TILES];
  float s[TILES];
#pragma unroll
  for (int k = 0; k < TILES; ++k) {
    if (k >= mine) break;  // uniform
    const int first = 16 * (wave + k * WAVES);
    auto page = [&](int i) {  // (behind the last page, that one again)
      return p.bounds + (int64_t)__shfl(id[k], first + i < n ? i : n - 1 - first) * p.record;
    };
#pragma unroll
    for (int m = 0; m < M; ++m)
      x[k].w[m] = *(const i32x4*)(page((col & ~(M - 1)) + m) + D / 2 * grp + 16 * (col & (M - 1)) + g * (2 * D));
    s[k] = ((const float*)(page(col) + Hkv * (2 * D)))[g];
  }
  __syncthreads();
  ScoreQuery<D> q;
  query_operand<D>(q, s_u[0], s_step);
#pragma unroll
  for (int k = 0; k < TILES; ++k) {
    if (k >= mine) break;  // uniform
    as_operands<M>(x[k]);
    i32x4 sum{0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < M; ++m) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.w[m], x[k].w[m], sum, 0, 0, 0);
    const float best = best_row(sum, q.step, p.group) * s[k];
    if (grp == 0) s_score[16 * (wave + k * WAVES) + col] = best;
  }
  __syncthreads();
  if (p.scores) {
    float* out = p.scores + (int64_t)seg * p.stride;
    for (int i = threadIdx.x; i < n; i += kSelectThreads) out[i] = s_score[i];
  }
  if (!all) choose_pages<1>(p, n, list, [&](int i) { return s_score[i]; });
}

// One launch takes 6 to 9 us for rows of up to 256 pages and 12 to 25 for 1,024, two take 11 to 18 and 15
// to 24, as long as a round of workgroups (one of 16 waves on a CU) has the batch; of short rows, two
// rounds are worth it too (64 rows, 8 KV heads, 128 pages: 13.1 and 15.9 us, 256 pages 19.1 and 19.7; 1,024
// pages 47.9 and 34.5, as bounds are read best with all heads of a page at once, which
// page_scores_kernel does).
bool select_at_once(const SelectParams& p, int cus) {
  const int64_t segs = (int64_t)p.num_seqs * p.num_kv_heads;
  return p.stride <= 256 ? segs <= 2 * cus : p.stride <= kSelectThreads && segs <= cus;
}

hipError_t launch_page_score_select(const SelectParams& p, hipStream_t s) {
  const dim3 grid((unsigned)(p.num_seqs * p.num_kv_heads));
  if (p.head_dim == 128)
    hipLaunchKernelGGL(page_score_select_kernel<128>, grid, dim3(kSelectThreads), 0, s, p);
  else
    hipLaunchKernelGGL(page_score_select_kernel<64>, grid, dim3(kSelectThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_page_scores(const SelectParams& p, int cus, hipStream_t s) {
  const int64_t most = (int64_t)p.num_seqs * ((p.stride + 15) / 16);  // tiles
  const dim3 grid((unsigned)(most < kScorePerCu * cus ? most : kScorePerCu * cus));
  if (p.head_dim == 128)
    hipLaunchKernelGGL(page_scores_kernel<128>, grid, dim3(64 * kScoreWaves), 0, s, p);
  else
    hipLaunchKernelGGL(page_scores_kernel<64>, grid, dim3(64 * kScoreWaves), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_page_select(const SelectParams& p, hipStream_t s) {
  // a thread's share of the longest row that the table holds
  const int items = (p.stride + kSelectThreads - 1) / kSelectThreads;
  const void* fn = items <= 1   ? (const void*)&page_select_kernel<1>
                   : items <= 2 ? (const void*)&page_select_kernel<2>
                   : items <= 4 ? (const void*)&page_select_kernel<4>
                   : items <= 8 ? (const void*)&page_select_kernel<8>
                   : items <= 16 ? (const void*)&page_select_kernel<16>
                                 : (const void*)&page_select_kernel<0>;
  SelectParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)(p.num_seqs * p.num_kv_heads)), dim3(kSelectThreads), args, 0, s);
}

}  // namespace dora
