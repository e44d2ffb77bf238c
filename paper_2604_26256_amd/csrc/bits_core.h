// The page step of the attentions that take some of a page's tokens (window, listed
// pages).  Included by HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode_core.h"
#include "tree_core.h"

namespace dora {

// A page of T tokens, of which those with a bit in `bits` count: scores, online
// softmax and weighted values for one tile of 16 query columns, as the plain decode's
// page step.  Values of tokens that do not count may be anything.  The V scale is folded into
// the weights as in the tree step, whose reasons hold here too.
template <int D, int T, bool FP8>
__device__ __forceinline__ void consume_bits(const PageRegs<D, T, FP8>& r, uint32_t bits,
                                             const TreeScale& vs, const bf16x8 (&qop)[D / 32],
                                             f32x4 (&acc)[D / 16], float& m_run, float& l_run) {
  constexpr int NT = T / 16, KSTEPS = D / 32, DBLK = D / 16;
  constexpr uint32_t ALL = T == 32 ? ~0u : 0xFFFFu;
  const int grp = (threadIdx.x & 63) >> 4;
  const bool some = bits != ALL;                // uniform
  const uint32_t own = bits >> (T / 4 * grp);  // this lane's T / 4 consecutive tokens
  f32x4 sc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      bf16x8 a;
      if constexpr (FP8) {
        const u32x4& wd = r.k[t * (D / 64) + (ks >> 1)];
        a = (ks & 1) ? fp8x8_to_bf16(wd[2], wd[3]) : fp8x8_to_bf16(wd[0], wd[1]);
      } else {
        a = __builtin_bit_cast(bf16x8, r.k[t * KSTEPS + ks]);
      }
      sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qop[ks], sc[t], 0, 0, 0);
    }
  }
  float mx = -__builtin_inff();
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x = FP8 ? __builtin_fmaf(sc[t][i], vs.mul, vs.add) : sc[t][i] * vs.mul;
      if (some && !((own >> (4 * t + i)) & 1u)) x = -__builtin_inff();
      sc[t][i] = x;
      mx = fmaxf(mx, x);
    }
  mx = max_xor32(max_xor16(mx));
  const float m_new = fmaxf(m_run, mx);
  const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
  m_run = m_new;
  float psum = 0.f;
  bf16x2 w[2 * NT];
#pragma unroll
  for (int t = 0; t < 2 * NT; ++t) {
    w[t] = bf16x2{(__bf16)__builtin_amdgcn_exp2f(sc[t >> 1][2 * (t & 1)] - m_new),
                  (__bf16)__builtin_amdgcn_exp2f(sc[t >> 1][2 * (t & 1) + 1] - m_new)};
    psum = __builtin_amdgcn_fdot2_f32_bf16(w[t], bf16x2{(__bf16)1.f, (__bf16)1.f}, psum, false);
  }
  if constexpr (FP8) {
    l_run = __builtin_fmaf(psum, vs.inv, l_run * alpha);
    if (__ballot(vs.left != 1.f)) {
#pragma unroll
      for (int t = 0; t < 2 * NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e)  // (a weight that does not count stays 0 under an infinity)
          if (!some || ((own >> (2 * t + e)) & 1u)) w[t][e] = (__bf16)((float)w[t][e] * vs.left);
    }
  } else {
    l_run = __builtin_fmaf(l_run, alpha, psum);
  }
  if (__ballot(alpha != 1.f)) {
#pragma unroll
    for (int i = 0; i < DBLK; ++i) acc[i] *= alpha;
  }
  if constexpr (T == 16) {
    const bf16x4 pb{w[0][0], w[0][1], w[1][0], w[1][1]};
#pragma unroll
    for (int i = 0; i < DBLK; ++i) {
      bf16x4 a;
      if constexpr (FP8)
        a = fp8x4_to_bf16(r.v[i]);
      else
        a = __builtin_bit_cast(bf16x4, r.v[i]);
      if (some) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!((own >> e) & 1u)) a[e] = (__bf16)0.f;
      }
      acc[i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, pb, acc[i], 0, 0, 0);
    }
  } else {
    const bf16x8 pb{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
#pragma unroll
    for (int i = 0; i < DBLK; ++i) {
      bf16x8 a;
      if constexpr (FP8)
        a = fp8x8_to_bf16(r.v[i][0], r.v[i][1]);
      else
        a = __builtin_bit_cast(bf16x8, r.v[i]);
      if (some) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((own >> e) & 1u)) a[e] = (__bf16)0.f;
      }
      acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb, acc[i], 0, 0, 0);
    }
  }
}

}  // namespace dora
