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
    return (uint32_t)(CODES + 2 * (group_slot(lane) + (lane & 15)));
  }

  typedef typename std::conditional<D == 128, u32x4, u32x2>::type kraw_t;
  struct Regs {
    kraw_t k[4];          // D / 4 dims of a token, of each sub-tile
    uint32_t ks;          // their exponents, a byte each
    u32x2 v[D / 16];      // 16 tokens of a dim
    uint16_t vs[D / 64];  // bf16 scales of token `lane & 15` of the lane's row group
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
      r.vs[h] = __builtin_nontemporal_load((const uint16_t*)(vt + vsoff + 2 * P * h));
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

  // The weights as an operand: each is rounded once, with its V scale, to bf16, as the matrix product wants it.
  // That is up to half a step, 2^-8 of a weight, so a result is off by no more than 2^-8 of sum w |v| / sum w;
  // against 64 bits results are off by 0.0022 of theirs, by their own rounding alone 0.0017.  The sums of
  // weights are of those before the rounding: a weight is rounded differently under each of its V scales, so that
  // no one sum of rounded ones would cancel it.
  // x times the value that lane U of the lane's row of 16 has in y.
  template <int U>
  static __device__ __forceinline__ float times_of(float x, float y) {
    return x * __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x150 + U, 0xF, 0xF, true));
  }
  template <int U>
  static __device__ __forceinline__ void scaled(bf16x8 (&w)[2], const f32x4 (&p)[4], float scale) {
    if constexpr (U < 16) {
      w[U >> 3][U & 7] = (__bf16)times_of<U>(p[U >> 2][U & 3], scale);
      scaled<U + 1>(w, p, scale);
    }
  }

  // The step: scores, softmax weights in the log2 domain, weighted values.  q(s): the query operand of
  // k-step s.  nv: of the 16 tokens of the
  // lane's row group those that count, the first nv; `all`: every lane's do (uniform).  What the other
  // slots hold is not used: a code is finite whatever it is, and scores and scales are replaced.
  //   m_run is a reference and not the running maximum: it moves only where a lane's weights sum to more than
  // kMostWeight, so that most steps neither look for their maximum nor rescale.
  //   What a row adds up stays below 2^128, whatever finite values it attends (and scores up to 2^24, from which on
  // fp32 holds no units of them): a lane's 16 weights sum to 2^8 at
  // most, so a row of up to 2^24 tokens adds at most 2^28 times 6 kFarScale, 2^126.6, for the steps whose V scales
  // are up to that; a step with a larger one has its reference kFarMargin above its largest score, so that such
  // tokens' weights are 2^-32 at most and add 2^24 * 2^-32 * 2^128.
  static constexpr float kMostWeight = 256.f;
  static constexpr float kFarScale = 0x1p96f, kFarMargin = 32.f;
  template <typename QueryAt>
  static __device__ __forceinline__ void consume(const Regs& r, bool all, int nv, float mul, QueryAt q,
                                                 f32x4 (&acc)[D / 16], float& m_run, float& l_run) {
    f32x4 sc[4], p[4];
    float ks[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      ks[t] = __uint_as_float(((r.ks >> (8 * t)) & 0xFFu) << 23);
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const bf16x8 row = q(s);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(r.k[t][s], ks[t]), row, sc[t], 0, 0, 0);
    }
    float scale[D / 64];
#pragma unroll
    for (int h = 0; h < D / 64; ++h) scale[h] = __uint_as_float((uint32_t)r.vs[h] << 16);
    if (!all) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * t + i >= nv) sc[t][i] = -__builtin_inff();
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
        if ((int)(threadIdx.x & 15) >= nv) scale[h] = 0.f;
    }
    float sum;
    auto weigh = [&]() {
      sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], mul, -m_run));
          sum += p[t][i];
        }
    };
    weigh();
    const bool far = fmaxf(scale[0], scale[D / 64 - 1]) > kFarScale;
    if (__ballot(far || !(sum <= kMostWeight))) {  // uniform
      const float margin = __ballot(far) ? kFarMargin : 0.f;
      float mx = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[t][i]);
      const float m_new = fmaxf(m_run, __builtin_fmaf(mul, max_xor32(max_xor16(mx)), margin));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[i] *= alpha;
      weigh();
    }
    l_run += sum;
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      bf16x8 w[2];
      scaled<0>(w, p, scale[h]);
#pragma unroll
      for (int i = 4 * h; i < 4 * h + 4; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(r.v[i][s], 1.0f), w[s], acc[i], 0, 0, 0);
    }
  }
};

}  // namespace dora
