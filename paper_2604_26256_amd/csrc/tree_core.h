// Device code that the tree attention kernels share: a sequence's stages, the range of
// a workgroup in the batch's list of them, and the step over 32 tokens.  Included by
// HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "decode_core.h"

namespace dora {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Smallest range of a workgroup, in stages.
constexpr int kTreeMinRange = 2;

// Stages of a sequence (steps of 32 tokens, steps_per_stage at a time): cache_stages over
// its cached tokens, then those of its drafts.  blocks: column blocks that have columns.
struct TreeSeq {
  int L, nodes, pages, cache_steps, cache_stages, stages, blocks;
};

__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b, int P, int steps_per_stage,
                                            int columns_per_block) {
  TreeSeq s;
  s.nodes = p.node_counts ? p.node_counts[b] : p.num_nodes;
  s.nodes = s.nodes < 0 ? 0 : s.nodes < p.num_nodes ? s.nodes : p.num_nodes;
  const int64_t most = (int64_t)p.stride * P;
  int L = p.seq_lens[b];
  L = L < 0 ? 0 : L;
  s.L = L < most ? L : (int)most;  // a contract violation stays in bounds
  s.pages = (s.L + P - 1) / P;
  s.cache_steps = (int)(((int64_t)s.L + 31) / 32);
  s.cache_stages = (s.cache_steps + steps_per_stage - 1) / steps_per_stage;
  const int draft_steps = (s.nodes + 31) / 32;
  s.stages = s.cache_stages + (draft_steps + steps_per_stage - 1) / steps_per_stage;
  s.blocks = (s.nodes * p.group + columns_per_block - 1) / columns_per_block;
  return s;
}

// This workgroup's place in the list of work.  Workgroups go to the 8 XCDs in turn; where rows are
// cut, each XCD gets one contiguous part of the list, so that the pieces of a segment are
// written and joined in one L2: 256 rows of 2,048 tokens at the median, fp8, 545 -> 524 us with 8
// nodes and 379 -> 371 with 4.  Not where rows are whole (128 of up to 2,048 tokens 43 -> 46:
// one XCD's can be longer than another's), nor with several column blocks (5 long rows, 2
// blocks, bf16, 154 -> 163).
__device__ __forceinline__ int tree_place(const TreeParams& p) {
  if (p.whole || p.blocks > 1) return (int)blockIdx.x;
  const int n = (int)gridDim.x, i = (int)blockIdx.x, each = n >> 3, more = n & 7, xcd = i & 7;
  return xcd * each + (xcd < more ? xcd : more) + (i >> 3);
}

// This workgroup's range [x0, x1) of the batch's `total` stages, cut for W workgroups, and
// the sequence b that holds x0.  Each segment counts as COST stages more than it has, in
// front of them, so that ranges of many short segments take no longer than others.  pre: LDS,
// [num_seqs + 1], the stages (over heads and blocks) before each sequence.
struct TreeRange {
  int x0, x1, total, W, b;
};

template <int P, int SP, int CB, int COST, int WAVES>
__device__ __forceinline__ TreeRange tree_range(const TreeParams& p, int place, int* pre) {
  __shared__ int s_wave[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), B = p.num_seqs;
  int carry = 0;
  for (int base = 0; base < B; base += 64 * WAVES) {
    int n = 0;
    if (base + tid < B) {
      const TreeSeq s = tree_seq(p, base + tid, P, SP, CB);
      n = s.blocks ? (s.stages + COST) * s.blocks * p.num_kv_heads : 0;
    }
    int incl = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += s_wave[w];
      carry += s_wave[w];
    }
    if (base + tid < B) pre[base + tid] = before + incl - n;
    __syncthreads();
  }
  if (tid == 0) pre[B] = carry;
  __syncthreads();
  TreeRange r;
  r.total = uni(carry);
  // Ranges of kTreeMinRange stages at least, none empty: the pieces of a cut segment are on
  // neighbouring workgroups.
  const int most = (r.total + kTreeMinRange - 1) / kTreeMinRange;
  r.W = most < (int)gridDim.x ? most : (int)gridDim.x;
  r.x0 = r.x1 = r.b = 0;
  if (place >= r.W) return r;
  r.x0 = (int)((int64_t)r.total * place / r.W);
  r.x1 = (int)((int64_t)r.total * (place + 1) / r.W);
  int lo = 0, hi = B;  // the last sequence with pre <= x0
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= r.x0) lo = mid; else hi = mid;
  }
  r.b = uni(lo);
  return r;
}

// Workgroups that hold pieces of a segment whose first piece is this workgroup's and whose
// last stage is `last`.
__device__ __forceinline__ int tree_pieces(const TreeRange& r, int place, int last) {
  int w = (int)((int64_t)last * r.W / r.total);  // near the range that holds `last`
  while (w + 1 < r.W && (int64_t)r.total * (w + 1) / r.W <= last) ++w;
  while ((int64_t)r.total * w / r.W > last) --w;
  return w - place + 1;
}

// What the 8 accumulator registers of a page's tokens are scaled by.  fp8: the page's V
// scale goes into the exponent, so that a weight is rounded once and the sum (over 2^add then)
// takes the rounded ones: for a row's largest weight the rounding cancels (with the scaling
// between the weight and its rounding the results were off by 0.0025 of their size against 64
// bits, by 0.0022 without; 0.0017 is the rounding of the result itself).  A V scale that has
// no such logarithm (0, negative, not finite, far from 1) stays a factor.  The logarithm and the
// reciprocal are the hardware's, each to about an ulp: over |log2| <= 40 the weights of a page are off by
// 2^-18 of their size at most, against sums that are off by 2^-23, far below the weights' own rounding.
struct TreeScale {
  float mul;   // scores
  float add;   // added to the scaled scores, log2 units
  float inv;   // 2^-add
  float left;  // what remains of the V scale: 1, or the scale itself
};

template <bool FP8>
__device__ __forceinline__ TreeScale tree_scale(float scale_log2, float k_scale, float v_scale) {
  if constexpr (!FP8) {
    return TreeScale{scale_log2, 0.f, 1.f, 1.f};
  } else {
    const bool fine = v_scale > 0x1p-40f && v_scale < 0x1p40f;
    const float add = fine ? __builtin_amdgcn_logf(v_scale) : 0.f;
    return TreeScale{scale_log2 * k_scale, add, fine ? __builtin_amdgcn_rcpf(v_scale) : 1.f,
                     fine ? 1.f : v_scale};
  }
}

// Weights above this (as a sum over a lane's 16 tokens) make a column's reference move up to
// its maximum.
constexpr float kTreeMostWeight = 256.f;

// Softmax weights of a step over 32 tokens for a tile of 32 columns: from the scores S^T = K Q^T,
// the weights 2^(s - m) of the log2 domain, rounded to bf16 for the product O^T += V^T P^T.  Lane
// (column lane & 31, half h = lane >> 5) holds in its registers 8s + e the scores of the 8
// tokens that it supplies to k-step s of the second product.  s0, s1: the scales of
// registers 0-7 and 8-15.  bits: the registers that count for the lane's column, where some
// does not (masked, uniform: a branch around the scores alone, as a second copy of the step
// would need registers for a second set of accumulators).
//   m is a reference and not the running maximum: it moves only where the weights grow past
// kTreeMostWeight, so that most steps neither look for their maximum nor rescale (96 of 175
// vector instructions a step, the matrix products apart).  Their sum is taken over the
// rounded weights: what the rounding does to a row's largest weight then cancels.
template <int D, bool FP8>
__device__ __forceinline__ void tree_weigh(f32x16& sc, TreeScale s0, TreeScale s1, bool masked,
                                           uint32_t bits, f32x16 (&acc)[D / 32], float& m_run,
                                           float& l_run, bf16x8 (&pb)[2]) {
  constexpr int DB = D / 32;
  if (masked) {
    asm volatile("" : "+v"(bits));  // (else the 16 tests are made before the branch, every step)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      sc[r] = (bits >> r) & 1u
                  ? (r < 8 ? __builtin_fmaf(sc[r], s0.mul, s0.add) : __builtin_fmaf(sc[r], s1.mul, s1.add))
                  : -__builtin_inff();
    s0.mul = s1.mul = 1.f;
    s0.add = s1.add = 0.f;
  }
  const float mul0 = s0.mul, mul1 = FP8 ? s1.mul : s0.mul;
  const float add0 = FP8 ? s0.add : 0.f, add1 = FP8 ? s1.add : 0.f;
  float sum[2];
  auto weigh = [&]() {
    const float b0 = add0 - m_run, b1 = add1 - m_run;
    sum[0] = sum[1] = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const bf16x2 w{
          (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], r < 8 ? mul0 : mul1, r < 8 ? b0 : b1)),
          (__bf16)__builtin_amdgcn_exp2f(
              __builtin_fmaf(sc[r + 1], r < 8 ? mul0 : mul1, r < 8 ? b0 : b1))};
      sum[r >> 3] = __builtin_amdgcn_fdot2_f32_bf16(w, bf16x2{(__bf16)1.f, (__bf16)1.f}, sum[r >> 3],
                                                    false);
      pb[r >> 3][r & 7] = w[0];
      pb[r >> 3][(r & 7) + 1] = w[1];
    }
  };
  weigh();
  if (__ballot(!(sum[0] + sum[1] <= kTreeMostWeight))) {
    float mx = -__builtin_inff();
#pragma unroll
    for (int r = 0; r < 16; ++r)
      mx = fmaxf(mx, __builtin_fmaf(sc[r], r < 8 ? mul0 : mul1, r < 8 ? add0 : add1));
    const float m_new = fmaxf(m_run, max_xor32(mx));
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
    weigh();
  }
  if constexpr (FP8) {
    l_run = __builtin_fmaf(sum[0], s0.inv, __builtin_fmaf(sum[1], s1.inv, l_run));
    if (s0.left != 1.f || s1.left != 1.f) {  // uniform
      if (!masked) bits = 0xFFFFu;
      asm volatile("" : "+v"(bits));
#pragma unroll
      for (int r = 0; r < 16; ++r)  // (a weight that does not count stays 0 under an infinity)
        if ((bits >> r) & 1u)
          pb[r >> 3][r & 7] = (__bf16)((float)pb[r >> 3][r & 7] * (r < 8 ? s0.left : s1.left));
    }
  } else {
    l_run += sum[0] + sum[1];
  }
}

// The whole step.  score(): the scores' tile, the last use of K; vf(i, s): V operand of head-dim
// rows 32i .. 32i + 31 and k-step s; scored(): called between the two.
template <int D, bool FP8, typename KF, typename SF, typename VF>
__device__ __forceinline__ void tree_step(KF score, SF scored, VF vf, TreeScale s0, TreeScale s1,
                                          bool masked, uint32_t bits, f32x16 (&acc)[D / 32],
                                          float& m_run, float& l_run) {
  f32x16 sc = score();
  scored();
  bf16x8 pb[2];
  tree_weigh<D, FP8>(sc, s0, s1, masked, bits, acc, m_run, l_run, pb);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int s = 0; s < 2; ++s)
      acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf(i, s), pb[s], acc[i], 0, 0, 0);
}

// Lane (row of K's tile or of V's, half h) and the 32 tokens of a step.  Register 8s + 4j +
// i of a lane is row 16s + 8j + 4h + i of the scores' tile; so that its 8 registers of
// k-step s are 8 consecutive tokens, row r holds token row_token(r).  Where a V row of a
// page is 32 bytes (fp8, 32 tokens), the lane's 16 tokens are consecutive: one 16-byte load.
template <int P, bool FP8>
struct TreeTokens {
  static constexpr bool RUN16 = FP8 && P == 32;
  static __device__ __forceinline__ int of_row(int r) {  // bits s j h i1 i0
    const int s = (r >> 4) & 1, j = (r >> 3) & 1, h = (r >> 2) & 1;
    return (RUN16 ? 16 * h + 8 * s : 16 * s + 8 * h) + 4 * j + (r & 3);
  }
  // Registers of half h whose tokens are among `bits`.
  static __device__ __forceinline__ uint32_t registers(uint32_t bits, int h) {
    if (RUN16) return (bits >> (16 * h)) & 0xFFFFu;
    return ((bits >> (8 * h)) & 0xFFu) | (((bits >> (16 + 8 * h)) & 0xFFu) << 8);
  }
};

// V's 16-byte pieces of 8 tokens in LDS (4 pieces a head-dim row) change places with the row,
// so that 16 rows' pieces of one column lie in different banks.
__device__ __forceinline__ int tree_v_at(int row, int piece) {
  return row * 64 + ((piece ^ ((row >> 2) & 3)) << 4);
}

// A step's K and V as a lane loads them: K in 16-byte pieces, V in 16 (8: fp8, 16 tokens)
// bytes per 32 head-dim rows and k-step (or both k-steps).
template <int D, int P, bool FP8>
struct TreeRegs {
  static constexpr int NK = FP8 ? D / 32 : D / 16;
  static constexpr bool RUN16 = TreeTokens<P, FP8>::RUN16;
  static constexpr int NV = (D / 32) * (RUN16 ? 1 : 2);
  typedef typename std::conditional<FP8 && !RUN16, u32x2, u32x4>::type vraw_t;
  u32x4 k[NK];
  vraw_t v[NV];
};

template <typename T>
__device__ __forceinline__ T tree_load(const uint8_t* at) {
  return __builtin_nontemporal_load((const T*)at);
}

// The V registers of a step whose tokens `own` alone count: the others, which may hold anything,
// become zeros.
template <int D, int P, bool FP8>
__device__ __forceinline__ void tree_keep(TreeRegs<D, P, FP8>& r, uint32_t own) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 keep;  // of the 8 tokens of k-step s: bf16 words, or (first two) fp8 words
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      keep[w] = 0;
#pragma unroll
      for (int e = 0; e < (FP8 ? 4 : 2); ++e) {
        constexpr int BITS = FP8 ? 8 : 16;
        const int tok = 8 * s + (FP8 ? 4 : 2) * w + e;
        if ((!FP8 || w < 2) && ((own >> tok) & 1u)) keep[w] |= ((1u << BITS) - 1u) << (BITS * e);
      }
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      if constexpr (TreeRegs<D, P, FP8>::RUN16) {
        r.v[i][2 * s] &= keep[0];
        r.v[i][2 * s + 1] &= keep[1];
      } else if constexpr (FP8) {
        r.v[2 * i + s] &= u32x2{keep[0], keep[1]};
      } else {
        r.v[2 * i + s] &= keep;
      }
    }
  }
}

// V's operands out of a step's registers.
template <int D, int P, bool FP8>
__device__ __forceinline__ bf16x8 tree_v(const TreeRegs<D, P, FP8>& r, int i, int s) {
  if constexpr (TreeRegs<D, P, FP8>::RUN16)
    return s ? fp8x8_to_bf16(r.v[i][2], r.v[i][3]) : fp8x8_to_bf16(r.v[i][0], r.v[i][1]);
  else if constexpr (FP8)
    return fp8x8_to_bf16(r.v[2 * i + s][0], r.v[2 * i + s][1]);
  else
    return __builtin_bit_cast(bf16x8, r.v[2 * i + s]);
}

// Head-dim offset of the 8 values that lane half h supplies to k-step s of the scores.  fp8: a
// lane's 16-byte K piece is 16 values, its k-steps 2m and 2m + 1.
template <bool FP8>
__device__ __forceinline__ int tree_dim(int s, int h) {
  return FP8 ? 16 * (2 * (s >> 1) + h) + 8 * (s & 1) : 16 * s + 8 * h;
}

// A lane's part of the queries, of column lane & 31: bf16 operands, or CODES.
template <int D, bool FP8, bool CODES>
struct TreeQuery {
  bf16x8 op[D / 16];
  __device__ __forceinline__ void load(const uint16_t* row, int h) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) op[s] = *(const bf16x8*)(row + tree_dim<FP8>(s, h));
  }
};

typedef int i32x8 __attribute__((ext_vector_type(8)));

// CODES: K's fp8 codes go into the products as they are, without the widening of each, so the
// queries are codes too, two for each value: q = 2^e (hi + lo / 16), e per column and 64 dims.  A
// bf16 value has 8 significant bits: hi is the nearest code, of 4, and what it leaves has 4 too, so
// the sum is exact but where lo is subnormal, and there off by 2^-14 2^e, 2^-21 of the largest of
// the 64 (an infinity or NaN makes all 64 NaN, as it makes the row).  Two fp8 products take the
// matrix pipe as long as the bf16 one does.
template <int D>
struct TreeQuery<D, true, true> {
  i32x8 hi[D / 64], lo[D / 64];
  int scales;  // bytes: 2^e of hi[0], lo[0], hi[1], lo[1], biased by 127
  __device__ __forceinline__ void load(const uint16_t* row, int h) {
    scales = 0;
#pragma unroll
    for (int m = 0; m < D / 64; ++m) {
      u32x4 w[4];  // the lane's K pieces 2m and 2m + 1
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = *(const u32x4*)(row + tree_dim<true>(4 * m + k, h));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a = w[k][i] & 0x7FFFu, c = (w[k][i] >> 16) & 0x7FFFu;
          top = top > a ? top : a;
          top = top > c ? top : c;
        }
      }
      const uint32_t there = (uint32_t)__shfl_xor((int)top, 32);  // the column's other values
      top = top > there ? top : there;
      // the largest becomes 128 to 255; be: its biased exponent, 14 to 255
      int be = (int)(top >> 7);
      be = be < 14 ? 14 : be;
      const float down = __uint_as_float((uint32_t)(261 - be) << 23);  // 2^-e, e = be - 134
      scales |= (int)((uint32_t)(be - 7) << (16 * m) | (uint32_t)(be - 11) << (16 * m + 8));
#pragma unroll
      for (int k = 0; k < 8; ++k) {  // 4 values each
        uint32_t a = 0, c = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const uint32_t v = w[k >> 1][2 * (k & 1) + p];
          const float x = __uint_as_float(v << 16) * down, y = __uint_as_float(v & 0xFFFF0000u) * down;
          if (p) {
            a = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, a, true);
            c = __builtin_amdgcn_cvt_pk_fp8_f32((x - __builtin_amdgcn_cvt_f32_fp8(a, 2)) * 16.f,
                                                (y - __builtin_amdgcn_cvt_f32_fp8(a, 3)) * 16.f, c, true);
          } else {
            a = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, a, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32((x - __builtin_amdgcn_cvt_f32_fp8(a, 0)) * 16.f,
                                                (y - __builtin_amdgcn_cvt_f32_fp8(a, 1)) * 16.f, c, false);
          }
        }
        hi[m][k] = top < 0x7F80u ? (int)a : 0x7F7F7F7F;
        lo[m][k] = (int)c;
      }
    }
  }
};

// Scores of a step's K for a tile of columns.
template <int D, int P, bool FP8, bool CODES>
__device__ __forceinline__ f32x16 tree_scores(const TreeRegs<D, P, FP8>& r,
                                              const TreeQuery<D, FP8, CODES>& q) {
  f32x16 sc;
#pragma unroll
  for (int i = 0; i < 16; ++i) sc[i] = 0.f;
  if constexpr (CODES) {
    constexpr int ONE = 127;  // 2^0
#pragma unroll
    for (int m = 0; m < D / 64; ++m) {
      const i32x8 k = __builtin_shufflevector(__builtin_bit_cast(i32x4, r.k[2 * m]),
                                              __builtin_bit_cast(i32x4, r.k[2 * m + 1]), 0, 1, 2, 3, 4, 5,
                                              6, 7);
      if (m == 0) {  // (the byte of the scales is a constant)
        sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.hi[m], sc, 0, 0, 0, ONE, 0, q.scales);
        sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.lo[m], sc, 0, 0, 0, ONE, 1, q.scales);
      } else {
        sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.hi[m], sc, 0, 0, 0, ONE, 2, q.scales);
        sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, q.lo[m], sc, 0, 0, 0, ONE, 3, q.scales);
      }
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      bf16x8 k;
      if constexpr (FP8) {
        const u32x4& w = r.k[ks >> 1];
        k = (ks & 1) ? fp8x8_to_bf16(w[2], w[3]) : fp8x8_to_bf16(w[0], w[1]);
      } else {
        k = __builtin_bit_cast(bf16x8, r.k[ks]);
      }
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.op[ks], sc, 0, 0, 0);
    }
  }
  return sc;
}

// Scores of 32 drafts: K row `key` of the lane, and for CODES the column's row of q, both bf16.
template <int D, bool FP8, bool CODES>
__device__ __forceinline__ f32x16 tree_draft_scores(const uint16_t* key, const uint16_t* row,
                                                    const TreeQuery<D, FP8, CODES>& q, int h) {
  f32x16 sc;
#pragma unroll
  for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int at = tree_dim<FP8>(s, h);
    bf16x8 op;
    if constexpr (CODES)
      op = *(const bf16x8*)(row + at);
    else
      op = q.op[s];
    sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(key + at), op, sc, 0, 0, 0);
  }
  return sc;
}

// Infinities and NaN in V of a draft belong to the nodes that attend it.  Among the operands of a
// product they would reach all of a tile's columns, since 0 x inf is NaN: so the products take zeros in
// their place, and where a piece has any (seldom) they are added to its results, once these are stored.

// V of 32 drafts from t0 on into LDS ([d][32 drafts], turned round), by THREADS threads, this one's
// part; whether a value in the wave's part is not finite (in the wave, uniform).
template <int D, int THREADS>
__device__ __forceinline__ bool tree_put_drafts(const TreeParams& p, uint8_t* vt, int b, int g, int t0,
                                                int nodes, int thread) {
  constexpr int PIECES = 32 * (D / 8) / THREADS;  // of a thread, 8 values each
  constexpr int BATCH = PIECES < 2 ? 1 : 2;       // loaded together
  static_assert(32 * (D / 8) % THREADS == 0 && PIECES % BATCH == 0, "whole batches");
  bool odd = false;
  while (true) {  // once, or twice where something is odd
    u16x2 top{0, 0};  // the largest magnitude's bits
#pragma unroll 1
    for (int k = 0; k < PIECES; k += BATCH) {
      u32x4 x[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int e = thread + THREADS * (k + j), t = e / (D / 8), ch = e - t * (D / 8);
        x[j] = u32x4{0u, 0u, 0u, 0u};
        if (t0 + t < nodes)
          x[j] = *(const u32x4*)(p.v_draft + (((int64_t)b * p.num_nodes + t0 + t) * p.num_kv_heads + g) * D + 8 * ch);
      }
      if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if ((x[j][i] & 0x7F80u) == 0x7F80u) x[j][i] &= 0xFFFF0000u;
            if ((x[j][i] & 0x7F800000u) == 0x7F800000u) x[j][i] &= 0xFFFFu;
          }
      }
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int e = thread + THREADS * (k + j), t = e / (D / 8), ch = e - t * (D / 8);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[j][i] & 0x7FFF7FFFu));
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *(uint16_t*)(vt + tree_v_at(8 * ch + i, t >> 3) + 2 * (t & 7)) =
              (uint16_t)(x[j][i >> 1] >> (16 * (i & 1)));
      }
    }
    if (__builtin_expect(!__any(top[0] >= 0x7F80 || top[1] >= 0x7F80), 1)) return odd;
    odd = true;
  }
}

// What the drafts that the lane's column attends (`sees`) add to its 4 values from head dim d0 on: the
// sum of their values that are not finite, else 0.
__device__ __forceinline__ f32x4 tree_odd_values(const TreeParams& p, int D, int b, int g, uint64_t sees,
                                                 int d0) {
  f32x4 sum{0.f, 0.f, 0.f, 0.f};
  for (; sees; sees &= sees - 1) {
    const int t = __builtin_ctzll(sees);
    const u32x2 w = *(const u32x2*)(p.v_draft + (((int64_t)b * p.num_nodes + t) * p.num_kv_heads + g) * D + d0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t v = (w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu;
      if ((v & 0x7F80u) == 0x7F80u) sum[e] += __uint_as_float(v << 16);
    }
  }
  return sum;
}

// Head dim of the first of a lane's 4 values in accumulator quad `quad`.
__device__ __forceinline__ int tree_quad_dim(int quad, int h) { return 32 * (quad >> 2) + 8 * (quad & 3) + 4 * h; }

// Adds tree_odd_values to a quad that this lane has stored: 4 outputs in bf16, or 4 values of a partial.
template <typename Quad>
__device__ __forceinline__ void tree_add_odd(Quad* at, f32x4 odd) {
  Quad o = *at;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (odd[e] != 0.f) o[e] = (float)o[e] + odd[e];
  *at = o;
}

}  // namespace dora
