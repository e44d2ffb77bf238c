// Device building blocks of attention over 4-bit pages: the register image of a step of 64
// tokens of one KV head, its loads, the query operand and the step.  Included by HIP
// sources only.
//
// A tile (one KV head of a page of P tokens) is 17/32 byte a value:
//   K  E2M1 codes [d / 32][P][32] (16 bytes a token and chunk, the even value in a byte's low
//      half), then the exponent of a power of two for each chunk of a token, biased by 127,
//      [d / 32][P / 16][4][4]: slot 16 a + 4 b + c at [a][c][b]
//   V  E2M1 codes [d][P] (P / 2 bytes a row), then a bf16 scale for each 64 dims of a token,
//      [d / 64][P]
// Both products are of bf16 operands, to which a code widens exactly.  K's power of two goes
// through the same conversion (a lane converts 32 dims of one token at a time), V's scale multiplies the
// weight of its token, as V's dims are rows of O^T += V^T P^T: so V's need not be a power of two, and
// one for 64 dims is as good as powers of two for 32 (the error of N(0, 1) values, relative: 0.106
// and 0.112).  (The scaled 16x16x128 product takes K's codes and powers of two as they are, but
// keeps few bits of products far below its largest: sums were off by 2^-12 of their terms where these
// spread, against 2^-24.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "decode_core.h"

namespace dora {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kFp4Step = 64;  // tokens

// MFMA row r of sub-tile t (of 4) is token 16 (r >> 2) + 4t + (r & 3) of the step, so that the
// scores of 16-lane row group `grp` are tokens 16 grp .. 16 grp + 15, those whose V the group's
// lanes hold.
template <int D, int P>
struct Fp4 {
  static constexpr int TILE = P * D / 32 * 17;
  static constexpr int CODES = P * D / 2;
  static constexpr int PAGES = kFp4Step / P;  // of a step

  // Which of the step's pages a lane reads K from, and V (and V's scales, and the tokens of its
  // scores) from.
  static __device__ __forceinline__ int k_page(int lane) { return (lane & 15) >> (P == 16 ? 2 : 3); }
  static __device__ __forceinline__ int v_page(int lane) { return lane >> (P == 16 ? 4 : 5); }
  // Slot of the first token of a lane's row group, in its page.
  static __device__ __forceinline__ int group_slot(int lane) {
    return P == 16 ? 0 : 16 * ((lane >> 4) & 1);
  }
  // Byte offsets in a tile.
  static __device__ __forceinline__ uint32_t k_off(int lane) {
    const int r = lane & 15, grp = lane >> 4;
    const uint32_t slot = (uint32_t)((P == 16 ? 0 : 16 * ((r >> 2) & 1)) + (r & 3));
    return D == 128 ? (grp * P + slot) * 16 : ((grp >> 1) * P + slot) * 16 + 8 * (grp & 1);
  }
  static __device__ __forceinline__ uint32_t k_scale_off(int lane) {
    const int r = lane & 15, chunk = D == 128 ? lane >> 4 : lane >> 5;
    return (uint32_t)(CODES + chunk * P + (P == 16 ? 0 : 16 * ((r >> 2) & 1)) + 4 * (r & 3));
  }
  static __device__ __forceinline__ uint32_t v_off(int lane) {
    return (uint32_t)((lane & 15) * (P / 2) + group_slot(lane) / 2);
  }
  static __device__ __forceinline__ uint32_t v_scale_off(int lane) {
    return (uint32_t)(CODES + 2 * group_slot(lane));
  }

  typedef typename std::conditional<D == 128, u32x4, u32x2>::type kraw_t;
  struct Regs {
    kraw_t k[4];          // D / 4 dims of a token, of each sub-tile
    uint32_t ks;          // their exponents, a byte each
    u32x2 v[D / 16];      // 16 tokens of a dim
    u32x4 vs[D / 64][2];  // bf16 scales of 16 tokens
  };

  // kt, vt: the lane's tiles.
  static __device__ __forceinline__ void load(Regs& r, const uint8_t* kt, const uint8_t* vt,
                                              uint32_t koff, uint32_t ksoff, uint32_t voff,
                                              uint32_t vsoff) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      r.k[t] = __builtin_nontemporal_load((const kraw_t*)(kt + koff + 64 * t));
    r.ks = __builtin_nontemporal_load((const uint32_t*)(kt + ksoff));
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      r.v[i] = __builtin_nontemporal_load((const u32x2*)(vt + voff + i * 8 * P));
#pragma unroll
    for (int h = 0; h < D / 64; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        r.vs[h][i] = __builtin_nontemporal_load((const u32x4*)(vt + vsoff + 2 * P * h + 16 * i));
  }

  // The query operand: a lane's values are those of the dims that it holds of K.
  typedef bf16x8 Query[D / 32];
  static __device__ __forceinline__ void load_query(Query& q, const uint16_t* qrow, bool valid) {
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      q[s] = valid ? *(const bf16x8*)(qrow + D / 4 * grp + 8 * s) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
  }

  static __device__ __forceinline__ bf16x8 widen(uint32_t w, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }

  // The step: scores, online softmax in the log2 domain, weighted values.  nv: of the 16
  // tokens of the lane's row group those that count, the first nv; `all`: every lane's do
  // (uniform).  What the other slots hold is not used: a code is finite whatever it is, and
  // scores and scaled weights are replaced.
  static __device__ __forceinline__ void consume(const Regs& r, bool all, int nv, float mul,
                                                 const Query& q, f32x4 (&acc)[D / 16],
                                                 float& m_run, float& l_run) {
    f32x4 sc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float scale = __uint_as_float(((r.ks >> (8 * t)) & 0xFFu) << 23);
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(r.k[t][s], scale), q[s], sc[t], 0, 0, 0);
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = sc[t][i] * mul;
        if (!all && 4 * t + i >= nv) x = -__builtin_inff();
        sc[t][i] = x;
        mx = fmaxf(mx, x);
      }
    mx = max_xor32(max_xor16(mx));
    const float m_new = fmaxf(m_run, mx);
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[t][i] = __builtin_amdgcn_exp2f(sc[t][i] - m_new);
        sum += sc[t][i];
      }
    l_run = __builtin_fmaf(l_run, alpha, sum);
    if (__ballot(alpha != 1.f)) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[i] *= alpha;
    }
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      bf16x8 w[2];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const uint32_t two = r.vs[h][u >> 3][(u >> 1) & 3];
        const float scale = __uint_as_float(u & 1 ? two & 0xFFFF0000u : two << 16);
        float x = sc[u >> 2][u & 3] * scale;
        if (!all && u >= nv) x = 0.f;
        w[u >> 3][u & 7] = (__bf16)x;
      }
#pragma unroll
      for (int i = 4 * h; i < 4 * h + 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(r.v[i][s], 1.0f), w[s], acc[i], 0, 0, 0);
    }
  }
};

}  // namespace dora
