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
//
// Bound by memory, and by more of it than the tokens: a token's V is one element of every
// head-dim row, so a page's V goes through whole whatever is new in it, and fp8 codes under
// a growing scale are read and written again.  1,024 paths of up to 16 tokens (8 KV heads of
// 128 dims): fp8 34 us for 133 MB that way (54 MB of tokens and codes alone), bf16 35 us; 24 runs
// of 300 to 700 tokens bf16 22 us (101 MB, 4.6 TB/s), fp8 30 us (76 MB).  fp8 also by the
// chain length -> page id -> scale and tokens -> scale's course -> tables -> codes, each
// step a trip to memory or a barrier, and by the encoding: 37 instructions a value through
// the division (whose ties sent most waves the long way round a cheaper test), 17 with
// path_codes8 (the same calls 65 -> 34 and 55 -> 30 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "fp8_core.h"
#include "path_core.h"

namespace dora {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPathMaxThreads = 512;

// bf16.  K: a thread stores one 16-byte chunk of one token, neighbours the slots of a
// chunk, non-temporally.  V: a thread takes 8 head-dim rows and 8 slots, turns them round
// in registers and stores 16 bytes a row, the slots that stay as they were read from the
// page.  Against the new slots' 2 bytes alone: 1,024 paths of up to 16 tokens (8 KV heads
// of 128 dims) 52 -> 35 us.  Plain K stores 40 us; non-temporal V stores 39, and 24
// prompts' runs of 300 to 700 tokens 36 us for 22 (15 at 6.6 TB/s).
__global__ __launch_bounds__(kPathMaxThreads) void append_path_bf16_kernel(PathParams p) {
  __shared__ int s_row[kPathMaxPage], s_bad;
  const int b = blockIdx.x, P = p.page_size, n = p.num_kv_heads * p.head_dim;
  const PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  if (!path_rows(p, pg, s_row, &s_bad)) return;
  const int nt = pg.hi - pg.lo;
  if (blockIdx.z == 0) {
    uint8_t* page = p.k_pages + pg.id * ((int64_t)n * P * 2);
    for (int e = threadIdx.x; e < nt * (n / 8); e += blockDim.x) {
      const int c = e / nt, i = e - c * nt;
      const u32x4 x =
          *(const u32x4*)(p.k_new + ((int64_t)b * p.num_tokens + s_row[i]) * n + 8 * c);
      __builtin_nontemporal_store(x, (u32x4*)(page + ((int64_t)c * P + pg.lo + i) * 16));
    }
    return;
  }
  uint8_t* page = p.v_pages + pg.id * ((int64_t)n * P * 2);
  const int g0 = pg.lo >> 3, groups = ((pg.hi + 7) >> 3) - g0;  // groups of 8 slots
  for (int e = threadIdx.x; e < groups * (n / 8); e += blockDim.x) {
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
    u32x4 old[8];
    uint32_t keep[4];  // of a row's 8 slots, those that stay
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 2 * i;
      keep[i] = (t >= pg.lo && t < pg.hi ? 0u : 0xFFFFu) |
                (t + 1 >= pg.lo && t + 1 < pg.hi ? 0u : 0xFFFF0000u);
    }
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      old[d] = u32x4{0u, 0u, 0u, 0u};
      if (!full) old[d] = *(const u32x4*)(page + ((int64_t)(8 * c + d) * P + t0) * 2);
    }
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      u32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __builtin_amdgcn_perm(x[2 * i + 1][d >> 1], x[2 * i][d >> 1],
                                     d & 1 ? 0x07060302 : 0x05040100);
        v[i] = (v[i] & ~keep[i]) | (old[d][i] & keep[i]);
      }
      *(u32x4*)(page + ((int64_t)(8 * c + d) * P + t0) * 2) = v;
    }
  }
}

// What a page's scale does over its new tokens: scale[i] is the one token i is encoded with,
// rcp[i] + rest[i] its reciprocal (rcp[i] = 0, and `exact` set, where only path_codes8_exact
// holds), after[i] the first growth (of `growths`) that comes after token i.
struct PathScales {
  float amax[kPathMaxPage];
  int nan[kPathMaxPage];
  float scale[kPathMaxPage], rcp[kPathMaxPage], rest[kPathMaxPage];
  float grow_from[kPathMaxPage], grow_to[kPathMaxPage];
  int after[kPathMaxPage];
  int growths, exact;
  int row[kPathMaxPage], bad;            // source rows, and whether one is none
  uint8_t lut[kPathMaxPage][256];        // row k: growths k, k + 1, ... one after the other
};

// The course of the scale, by the first wave: lane i has token i.  s0: the page's scale before.
//   s_i = max(s0, fresh_0 .. fresh_i), and token i makes it grow where its fresh scale is larger
// than all before (an unset, NaN scale is below every other).
__device__ __forceinline__ float path_scales(PathScales& sc, const PathPage& pg, float s0) {
  const int i = threadIdx.x, nt = pg.hi - pg.lo;
  const float fresh = i < nt ? fmaxf(__fdiv_rn(sc.amax[i], 448.0f), 0x1p-126f) : 0.f;
  float top = fresh;
#pragma unroll
  for (int off = 1; off < kPathMaxPage; off <<= 1) {
    const float y = __shfl_up(top, off);
    if (i >= off) top = fmaxf(top, y);
  }
  const float known = pg.lo > 0 && s0 == s0 ? s0 : 0.f;  // (fresh scales are positive)
  float before = __shfl_up(top, 1);
  before = i == 0 ? known : fmaxf(known, before);
  const bool first = pg.lo == 0 && i == 0;  // slot 0 sets the scale
  const bool grow = i < nt && !first && !(fresh <= before);
  const uint64_t grows = __ballot(grow);
  const int k = __popcll(grows & ((1ull << i) - 1));
  const float s = fmaxf(before, fresh);
  if (grow) {
    sc.grow_from[k] = i == 0 ? s0 : before;  // (i = 0: NaN where the scale was unset)
    sc.grow_to[k] = fresh;
  }
  const bool quick = s > 0x1p-80f && s < 0x1p100f && !(i < nt && sc.nan[i]);
  if (i < nt) {
    const float rcp = quick ? __fdiv_rn(1.0f, s) : 0.f;
    sc.scale[i] = s;
    sc.rcp[i] = rcp;
    sc.rest[i] = fmaf(-s, rcp, 1.0f) * rcp;
    sc.after[i] = k + (grow ? 1 : 0);
  }
  const bool exact = __any(i < nt && !quick);
  if (i == 0) {
    sc.growths = __popcll(grows);
    sc.exact = exact;
  }
  return __shfl(s, nt - 1);
}

// Codes of 8 bf16 values w over scale s, as the nearest E4M3FN code of the quotient rounded to fp32.
__device__ __forceinline__ u32x2 path_codes8_exact(u32x4 w, float s) {
  u32x2 out{0u, 0u};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    out[k >> 1] |= f32_to_e4m3(__fdiv_rn(bf16_bits_to_f32((uint16_t)w[k]), s)) << (16 * (k & 1));
    out[k >> 1] |= f32_to_e4m3(__fdiv_rn(bf16_bits_to_f32((uint16_t)(w[k] >> 16)), s))
                   << (16 * (k & 1) + 8);
  }
  return out;
}

// The same with rcp + rest = 1 / s to 2^-47 and rcp = 1 / s rounded, for finite values of at most
// 448 s and 2^-80 < s < 2^100:
//   q = x rcp + x rest is next to the quotient, r = x - q s is exact, and q + r rcp, rounded, is
// the rounded quotient (Markstein; what is too small for an exact r has code 0 either way).  The
// hardware's conversion and f32_to_e4m3 agree on all values up to 463.  A quotient of -0 comes out
// +0, so the signs are x's own.  6 instructions a value; the division alone is 12.
__device__ __forceinline__ u32x2 path_codes8(u32x4 w, float s, float rcp, float rest) {
  u32x2 out{0u, 0u};
  auto over = [&](float x) {
    const float q = fmaf(x, rcp, x * rest);
    return fmaf(fmaf(-q, s, x), rcp, q);
  };
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = over(__uint_as_float(w[k] << 16)), b = over(__uint_as_float(w[k] & 0xFFFF0000u));
    if (k & 1)
      out[k >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, out[k >> 1], true);
    else
      out[k >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, out[k >> 1], false);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    out[i] = (out[i] & 0x7F7F7F7Fu) |
             (__builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07050301) & 0x80808080u);
  return out;
}

// Four codes through a table.
__device__ __forceinline__ uint32_t path_map4(uint32_t w, const uint8_t* lut) {
  return lut[w & 0xFF] | (uint32_t)lut[(w >> 8) & 0xFF] << 8 | (uint32_t)lut[(w >> 16) & 0xFF] << 16 |
         (uint32_t)lut[w >> 24] << 24;
}

// 4 x 4 bytes turned round: byte j of r[i] to byte i of r[j].
__device__ __forceinline__ void path_turn4(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602);
  a = __builtin_amdgcn_perm(cd0, ab0, 0x05040100);
  b = __builtin_amdgcn_perm(cd0, ab0, 0x07060302);
  c = __builtin_amdgcn_perm(cd1, ab1, 0x05040100);
  d = __builtin_amdgcn_perm(cd1, ab1, 0x07060302);
}

constexpr int kPathBatch = 4;  // pieces whose loads a thread issues together
template <bool IS_K>
__device__ __forceinline__ void path_side(const PathParams& p, uint8_t* pages, float* scales,
                                          const uint16_t* token, PathScales& sc) {
  int* s_row = sc.row;
  uint8_t(*lut)[256] = sc.lut;
  const int b = blockIdx.x, P = p.page_size, n = p.num_kv_heads * p.head_dim, tid = threadIdx.x;
  const int T = blockDim.x;
  const PathPage pg = path_page(p, b, blockIdx.y);
  if (pg.id < 0) return;  // uniform
  const float s0 = scales[pg.id];  // (before path_rows' barriers; stored after them, by one thread)
  if (!path_rows(p, pg, s_row, &sc.bad)) return;
  const int nt = pg.hi - pg.lo;
  const uint16_t* __restrict__ src = token + (int64_t)b * p.num_tokens * n;
  // a wave per token, two at a time: its largest magnitude
  const int waves = T >> 6;
  for (int i = tid >> 6; i < nt; i += 2 * waves) {
    const int j = i + waves < nt ? i + waves : i;
    const uint16_t* x = src + (int64_t)s_row[i] * n;
    const uint16_t* y = src + (int64_t)s_row[j] * n;
    u16x2 m{0, 0}, m2{0, 0};  // the magnitudes' bits order as the magnitudes do
#pragma unroll 2
    for (int e = 8 * (tid & 63); e < n; e += 8 * 64) {
      const u32x4 w = *(const u32x4*)(x + e), v = *(const u32x4*)(y + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[k] & 0x7FFF7FFFu));
        m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, v[k] & 0x7FFF7FFFu));
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      m = __builtin_elementwise_max(
          m, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, m), off)));
      m2 = __builtin_elementwise_max(
          m2, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, m2), off)));
    }
    const int top = m[0] > m[1] ? m[0] : m[1], top2 = m2[0] > m2[1] ? m2[0] : m2[1];
    if ((tid & 63) == 0) {
      sc.amax[i] = bf16_bits_to_f32((uint16_t)top);
      sc.amax[j] = bf16_bits_to_f32((uint16_t)top2);
      sc.nan[i] = top > 0x7F80;
      sc.nan[j] = top2 > 0x7F80;
    }
    for (int u = i; top > 0x7F80 || top2 > 0x7F80; u = j) {  // a NaN: the largest of the others
      float f = 0.f;
      for (int e = tid & 63; e < n; e += 64)
        f = fmaxf(f, fabsf(bf16_bits_to_f32(src[(int64_t)s_row[u] * n + e])));
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) f = fmaxf(f, __shfl_xor(f, off));
      if ((tid & 63) == 0) sc.amax[u] = f;
      if (u == j) break;
    }
  }
  __syncthreads();
  if (tid < 64) {
    const float s = path_scales(sc, pg, s0);
    if (tid == 0) scales[pg.id] = s;
  }
  __syncthreads();
  const int growths = sc.growths;
  for (int k = growths - 1; k >= 0; --k) {
    if (tid < 256) {
      const uint8_t c = (uint8_t)f32_to_e4m3(
          __fdiv_rn(e4m3_to_f32((uint32_t)tid) * sc.grow_from[k], sc.grow_to[k]));
      lut[k][tid] = k == growths - 1 ? c : lut[k + 1][c];
    }
    __syncthreads();
  }
  uint8_t* __restrict__ page = pages + pg.id * ((int64_t)n * P);
  // Codes of 8 values w of token i after all of the page's growths.
  const bool exact = sc.exact;
  auto after = [&](u32x2 c, int i) {
    const int k = sc.after[i];
    if (k < growths) c = u32x2{path_map4(c[0], lut[k]), path_map4(c[1], lut[k])};
    return c;
  };
  if constexpr (IS_K) {
    // old slots, where they change: 16-byte pieces (16-dim chunk, slot)
    const int old = growths ? pg.lo * (n / 16) : 0;
    for (int e0 = tid; e0 < old; e0 += kPathBatch * T) {
      u32x4 w[kPathBatch];
      u32x4* at[kPathBatch];
#pragma unroll
      for (int i = 0; i < kPathBatch; ++i) {
        int e = e0 + i * T;
        e = e < old ? e : e0;  // past the end: the first piece again, not stored
        const int c = e / pg.lo, t = e - c * pg.lo;
        at[i] = (u32x4*)(page + ((int64_t)c * P + t) * 16);
        w[i] = *at[i];
      }
#pragma unroll
      for (int i = 0; i < kPathBatch; ++i)
        if (e0 + i * T < old)
          *at[i] = u32x4{path_map4(w[i][0], lut[0]), path_map4(w[i][1], lut[0]),
                         path_map4(w[i][2], lut[0]), path_map4(w[i][3], lut[0])};
    }
#pragma unroll 2
    for (int e = tid; e < nt * (n / 16); e += T) {
      const int c = e / nt, i = e - c * nt;
      const u32x4* x = (const u32x4*)(src + (int64_t)s_row[i] * n + 16 * c);
      const u32x4 w0 = x[0], w1 = x[1];
      const float s = sc.scale[i], rcp = sc.rcp[i], rest = sc.rest[i];
      u32x2 c0 = path_codes8(w0, s, rcp, rest), c1 = path_codes8(w1, s, rcp, rest);
      if (exact && rcp == 0.f) {
        c0 = path_codes8_exact(w0, s);
        c1 = path_codes8_exact(w1, s);
      }
      c0 = after(c0, i);
      c1 = after(c1, i);
      *(u32x4*)(page + ((int64_t)c * P + pg.lo + i) * 16) = u32x4{c0[0], c0[1], c1[0], c1[1]};
    }
  } else {
    // a thread per 8 rows and 8 slots; what is not new is read, mapped and stored again
    const int g0 = growths ? 0 : pg.lo >> 3, groups = ((pg.hi + 7) >> 3) - g0;
    for (int e = tid; e < groups * (n / 8); e += T) {
      const int c = e / groups, t0 = 8 * (g0 + e - c * groups);
      const bool full = t0 >= pg.lo && t0 + 8 <= pg.hi;
      u32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // all loads first
        const int t = t0 + i;
        x[i] = u32x4{0u, 0u, 0u, 0u};
        if (t >= pg.lo && t < pg.hi)
          x[i] = *(const u32x4*)(src + (int64_t)s_row[t - pg.lo] * n + 8 * c);
      }
      uint32_t cd[8][2];  // codes of slot i: 8 rows
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = t0 + i;
        cd[i][0] = cd[i][1] = 0u;
        if (t >= pg.lo && t < pg.hi) {
          const int j = t - pg.lo;
          const u32x2 q = after(path_codes8(x[i], sc.scale[j], sc.rcp[j], sc.rest[j]), j);
          cd[i][0] = q[0];
          cd[i][1] = q[1];
        }
      }
      if (exact) {
#pragma unroll 1
        for (int t = t0 > pg.lo ? t0 : pg.lo; t < t0 + 8 && t < pg.hi; ++t) {
          const int j = t - pg.lo;
          if (sc.rcp[j] != 0.f) continue;
          const u32x4 w = *(const u32x4*)(src + (int64_t)s_row[j] * n + 8 * c);
          const u32x2 q = after(path_codes8_exact(w, sc.scale[j]), j);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (t0 + i == t) {
              cd[i][0] = q[0];
              cd[i][1] = q[1];
            }
        }
      }
      u32x2 out[8];
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        out[d] = u32x2{0u, 0u};
        if (!full) out[d] = *(const u32x2*)(page + (int64_t)(8 * c + d) * P + t0);
      }
      // bytes of a row's 8 slots that stay, and whether they are mapped
      const int below = pg.lo - t0, upto = pg.hi - t0;
      const uint64_t lowmask = below <= 0 ? 0ull : below >= 8 ? ~0ull : (1ull << (8 * below)) - 1;
      const uint64_t highmask = upto >= 8 ? 0ull : upto <= 0 ? ~0ull : ~((1ull << (8 * upto)) - 1);
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        if (full) break;
        const uint64_t w = (uint64_t)out[d][1] << 32 | out[d][0];
        uint64_t low = w & lowmask;
        if (growths && lowmask) {
          low = ((uint64_t)path_map4(out[d][1], lut[0]) << 32 | path_map4(out[d][0], lut[0])) & lowmask;
        }
        const uint64_t keep = low | (w & highmask);
        out[d] = u32x2{(uint32_t)keep, (uint32_t)(keep >> 32)};
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {  // rows 4r .. 4r + 3
        path_turn4(cd[0][r], cd[1][r], cd[2][r], cd[3][r]);
        path_turn4(cd[4][r], cd[5][r], cd[6][r], cd[7][r]);
      }
#pragma unroll
      for (int d = 0; d < 8; ++d)
        *(u32x2*)(page + (int64_t)(8 * c + d) * P + t0) =
            out[d] | u32x2{cd[d & 3][d >> 2], cd[4 + (d & 3)][d >> 2]};
    }
  }
}

__global__ __launch_bounds__(kPathMaxThreads) void append_path_fp8_kernel(PathParams p) {
  __shared__ PathScales sc;
  if (blockIdx.z == 0)
    path_side<true>(p, p.k_pages, p.k_scales, p.k_new, sc);
  else
    path_side<false>(p, p.v_pages, p.v_scales, p.v_new, sc);
}

hipError_t launch_append_path(const PathParams& p, bool fp8, hipStream_t s) {
  if (p.dev_status) {
    const hipError_t e = launch_fill_i32(p.dev_status, (int32_t)DORA_OK, 1, s);
    if (e != hipSuccess) return e;
  }
  // pages that p.num_tokens tokens can touch
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const dim3 grid((unsigned)p.num_seqs, pages, 2);
  // fp8: 512 threads where the grid leaves CUs to spare (64 paths of up to 64 tokens, 8 KV heads of
  // 128 dims, 16.8 us against 19.4 at 256 threads; one token of each of 256 sequences, 17.3 against
  // 19.0), else 256, so that more pages are under way (1,024 paths of up to 16 tokens 34.4 against
  // 38.2 at 512; 24 runs of 300 to 700 tokens 30.1 against 31.8).  bf16: 256 (22 against 23).
  const int threads = fp8 && (int64_t)p.num_seqs * pages * 2 < 1024 ? 512 : 256;
  if (fp8)
    hipLaunchKernelGGL(append_path_fp8_kernel, grid, dim3(threads), 0, s, p);
  else
    hipLaunchKernelGGL(append_path_bf16_kernel, grid, dim3(threads), 0, s, p);
  return hipGetLastError();
}

}  // namespace dora
