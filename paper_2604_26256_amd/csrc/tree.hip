// Decode attention for a tree of drafted tokens per sequence, over the paged cache
// and the drafts' own keys and values.  All nodes of a sequence see its whole cache,
// so every cached byte is read once and applied to the C = nodes x group columns of
// its KV head; among the drafts a column sees what its node's mask says.
//
//   scores  S^T = K Q^T, softmax weights 2^(s - m) with a running maximum, O^T += V^T P^T
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "decode_core.h"

namespace dora {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Pages whose ids (and fp8 scales) a workgroup holds in LDS at a time.
constexpr int kTreeWindow = 512;
// Smallest range of a workgroup, in stages.
constexpr int kTreeMinRange = 2;

// Stages of a sequence: cache_stages over its pages, then those of its drafts.
struct TreeSeq {
  int L, nodes, pages, cache_steps, cache_stages, stages, blocks;
};

// Row of a 32-token tile that holds token t, and the other way round (bits 2 and 3
// change places): the rows of a lane's accumulator, 8j + 4h + i, then are the tokens
// 16s + 8h + 4(j & 1) + i, which are the 8 consecutive tokens of k-step s that this
// lane supplies to the second product.
__device__ __forceinline__ int tree_row(int t) {
  return (t & 0x13) | ((t & 4) << 1) | ((t & 8) >> 1);
}

// V's 16-byte pieces (8 tokens of a head-dim row, 4 pieces a row) change places with
// the row so that 16 rows' pieces of one column lie in different banks.
__device__ __forceinline__ int tree_v_at(int row, int piece) {
  return row * 64 + ((piece ^ ((row >> 2) & 3)) << 4);
}

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

// NT tiles of 32 columns are held by a team of NT waves; SP = 4 / NT teams take the
// 32-token steps of a stage in turn.  A workgroup takes an equal, contiguous range of
// the batch's (sequence, KV head, column block, stage) list, as the plain decode's
// wavefronts do, or, where p.whole, one (sequence, KV head, column block).
//   A stage's pages go HBM -> registers (two stages in flight) -> LDS, fp8 widened to
// bf16 on the way, so that a team's waves share one read and one conversion.
template <int D, int P, bool FP8, int NT>
__global__ __launch_bounds__(64 * kTreeWaves, NT == 1 ? 1 : 2) void tree_kernel(TreeParams p) {
  constexpr int SP = kTreeWaves / NT, TT = 64 * NT, PAIR = 32 / P;
  constexpr int KS = D / 16, DB = D / 32, CB = 32 * NT;
  constexpr int TILE = P * D * (FP8 ? 1 : 2);            // bytes of one (page, KV head) tile
  constexpr int NK = 32 * D * (FP8 ? 1 : 2) / 16;        // 16-byte pieces of a step's K (V: as many)
  constexpr int PER = 2 * NK / TT;                       // pieces of a thread
  constexpr int KB = 32 * D * 2;                         // LDS bytes of a step's K (V: as many)
  static_assert(2 * NK % TT == 0, "every thread has as many pieces");
  __shared__ __align__(16) uint8_t s_kv[2][SP][2 * KB];
  __shared__ int s_pid[kTreeWindow];
  __shared__ float s_ksc[FP8 ? kTreeWindow : 1], s_vsc[FP8 ? kTreeWindow : 1];
  __shared__ float2 s_ml[kTreeWaves][32];
  __shared__ int s_wave[kTreeWaves];
  extern __shared__ int s_pre[];  // stages (over heads and blocks) before each sequence, [B + 1]

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int team = wave / NT, tile = wave % NT, tt = tid - team * TT;
  const int B = p.num_seqs, Hkv = p.num_kv_heads, G = p.group;

  int x0 = 0, x1 = 0, total = 0, W = 1;
  int b = 0;
  if (p.whole) {
    b = (int)blockIdx.x / (Hkv * p.blocks);
  } else {
    int carry = 0;
    for (int base = 0; base < B; base += 64 * kTreeWaves) {
      int n = 0;
      if (base + tid < B) {
        const TreeSeq s = tree_seq(p, base + tid, P, SP, CB);
        n = s.stages * s.blocks * Hkv;
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
      for (int w = 0; w < kTreeWaves; ++w) {
        if (w < wave) before += s_wave[w];
        carry += s_wave[w];
      }
      if (base + tid < B) s_pre[base + tid] = before + incl - n;
      __syncthreads();
    }
    if (tid == 0) s_pre[B] = carry;
    __syncthreads();
    total = uni(carry);
    // Ranges of kTreeMinRange stages at least, none empty: the pieces of a cut segment
    // are on neighbouring workgroups.
    W = (total + kTreeMinRange - 1) / kTreeMinRange;
    W = W < (int)gridDim.x ? W : (int)gridDim.x;
    if (tid == 0) p.cuts[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if ((int)blockIdx.x >= W) return;  // uniform
    x0 = (int)((int64_t)total * blockIdx.x / W);
    x1 = (int)((int64_t)total * (blockIdx.x + 1) / W);
    int lo = 0, hi = B;    // the sequence that holds x0: the last with s_pre <= x0
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_pre[mid] <= x0) lo = mid; else hi = mid;
    }
    b = uni(lo);
  }

  bool first_piece = true;
  int x = x0;
  while (true) {
    // the piece: stages a .. z - 1 of (b, g, block)
    const TreeSeq sq = tree_seq(p, b, P, SP, CB);
    int g, blk, a, z;
    if (p.whole) {
      const int r = (int)blockIdx.x - b * Hkv * p.blocks;
      g = r / p.blocks;
      blk = r - g * p.blocks;
      a = 0;
      z = sq.stages;
      if (blk >= sq.blocks) return;  // uniform: no such columns (or no nodes)
    } else {
      const int r = x - s_pre[b];
      const int gb = r / sq.stages;
      g = gb / sq.blocks;
      blk = gb - g * sq.blocks;
      a = r - gb * sq.stages;
      z = sq.stages - a < x1 - x ? sq.stages : a + (x1 - x);
    }
    g = uni(g);
    blk = uni(blk);
    a = uni(a);
    z = uni(z);
    const int n_pages = uni(sq.pages), L = uni(sq.L), nodes = uni(sq.nodes);
    const int cache_steps = uni(sq.cache_steps), cache_stages = uni(sq.cache_stages);

    // query operand: this lane's column
    const int c = blk * CB + tile * 32 + col;
    const int node = c / G, head = c - node * G;
    const bool mine = node < nodes;
    const int64_t row = (((int64_t)b * p.num_nodes + (mine ? node : 0)) * p.num_q_heads +
                         (int64_t)g * G + (mine ? head : 0));
    bf16x8 qop[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qop[s] = *(const bf16x8*)(p.q + row * D + 16 * s + 8 * h);
      if (!mine) qop[s] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    const uint64_t live = nodes >= 64 ? ~0ull : (1ull << nodes) - 1;
    const uint64_t sees = mine ? p.tree_mask[(int64_t)b * p.num_nodes + node] & live : 0ull;
    const bool active = uni(blk * CB + tile * 32 < nodes * G);  // the wave's tile has columns

    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    float m_run = kNoMax, l_run = 0.f;

    // One step from LDS.  bits: tokens that count (of this lane's column); all: no masks.
    auto consume = [&](const uint8_t* kv, uint32_t bits, bool all, float ks0, float ks1, float vs0,
                       float vs1) {
      f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 kf = *(const bf16x8*)(kv + ((2 * s + h) * 32 + col) * 16);
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qop[s], sc, 0, 0, 0);
      }
      float mx = -__builtin_inff();
      const uint32_t own = bits >> (8 * h);  // register r = 8s + 4jj + i: bit 16s + 4jj + i
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] *= r < 8 ? ks0 : ks1;
        if (!all && !((own >> (16 * (r >> 3) + (r & 7))) & 1u)) sc[r] = -__builtin_inff();
        mx = fmaxf(mx, sc[r]);
      }
      mx = max_xor32(mx);
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      float sum = 0.f;
      bf16x8 pb[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(sc[r] - m_new);
        sum += e;
        pb[r >> 3][r & 7] = (__bf16)(FP8 ? e * (r < 8 ? vs0 : vs1) : e);
      }
      l_run = l_run * alpha + sum;
      if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const bf16x8 vf = *(const bf16x8*)(kv + KB + tree_v_at(32 * i + col, 2 * s + h));
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[s], acc[i], 0, 0, 0);
        }
    };

    // Cached tokens, in windows of the pages whose ids fit the LDS array.
    constexpr int WST = kTreeWindow / (PAIR * SP);  // stages of a window
    const int c_end = z < cache_stages ? z : cache_stages;
    for (int w0 = a; w0 < c_end; w0 += WST) {
      const int n_st = c_end - w0 < WST ? c_end - w0 : WST;
      const int j0 = w0 * SP * PAIR;
      const int n_win = n_pages - j0 < kTreeWindow ? n_pages - j0 : kTreeWindow;
      __syncthreads();  // the arrays and the buffers are free
      for (int t = tid; t < n_win; t += 64 * kTreeWaves) {
        const int pid = p.block_table[(int64_t)b * p.stride + j0 + t];
        s_pid[t] = pid;
        if constexpr (FP8) {
          s_ksc[t] = p.scale_log2 * p.k_scales[pid];
          s_vsc[t] = p.v_scales[pid];
        }
      }
      __syncthreads();
      // Stage w0 + u of this thread's team; past the end the last page's pieces again.
      auto load = [&](u32x4 (&r)[PER], int u) {
        const int step0 = (u * SP + team) * PAIR;  // first page, from j0
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int e = tt + k * TT;
          const bool is_v = e >= NK;
          const int idx = is_v ? e - NK : e;
          const int pg = PAIR == 2 ? idx / (NK / 2) : 0, rem = PAIR == 2 ? idx - pg * (NK / 2) : idx;
          const int at = step0 + pg < n_win ? step0 + pg : n_win - 1;
          const uint8_t* base = is_v ? p.v_pages : p.k_pages;
          r[k] = __builtin_nontemporal_load(
              (const u32x4*)(base + (int64_t)s_pid[at] * p.page_bytes + (int64_t)g * TILE + rem * 16));
        }
      };
      auto store = [&](const u32x4 (&r)[PER], int u, int buf) {
        uint8_t* kv = s_kv[buf][team];
        const int nv = L - ((w0 + u) * SP + team) * 32;  // tokens of the step that count
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int e = tt + k * TT;
          const bool is_v = e >= NK;
          const int idx = is_v ? e - NK : e;
          const int pg = PAIR == 2 ? idx / (NK / 2) : 0, rem = PAIR == 2 ? idx - pg * (NK / 2) : idx;
          u32x4 w = r[k];
          if (!is_v) {
            const int ch = rem / P, row_ = tree_row(pg * P + rem % P);
            if constexpr (FP8) {
              *(bf16x8*)(kv + ((2 * ch) * 32 + row_) * 16) = fp8x8_to_bf16(w[0], w[1]);
              *(bf16x8*)(kv + ((2 * ch + 1) * 32 + row_) * 16) = fp8x8_to_bf16(w[2], w[3]);
            } else {
              *(u32x4*)(kv + (ch * 32 + row_) * 16) = w;
            }
          } else {
            constexpr int TOK = FP8 ? 16 : 8, PR = P / TOK;  // tokens of a piece, pieces of a page's row
            const int d = rem / PR, q = pg * PR + rem % PR;
            if (nv < 32) {  // uniform in the team: slots past the sequence hold anything
              const int keep = nv - q * TOK;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int left = keep - i * (TOK / 4);
                uint32_t m = 0;
                if (left >= TOK / 4) m = ~0u;
                else if (left > 0) m = (1u << (left * (FP8 ? 8 : 16))) - 1u;
                w[i] &= m;
              }
            }
            if constexpr (FP8) {
              *(bf16x8*)(kv + KB + tree_v_at(d, 2 * q)) = fp8x8_to_bf16(w[0], w[1]);
              *(bf16x8*)(kv + KB + tree_v_at(d, 2 * q + 1)) = fp8x8_to_bf16(w[2], w[3]);
            } else {
              *(u32x4*)(kv + KB + tree_v_at(d, q)) = w;
            }
          }
        }
      };
      auto compute = [&](int u, int buf) {
        const int step = (w0 + u) * SP + team;
        if (!active || step >= cache_steps) return;
        const int nv = L - step * 32;
        float ks0 = p.scale_log2, ks1 = ks0, vs0 = 1.f, vs1 = 1.f;
        if constexpr (FP8) {
          const int at = (u * SP + team) * PAIR;
          const int at1 = PAIR == 2 && at + 1 < n_win ? at + 1 : at;
          ks0 = s_ksc[at];
          vs0 = s_vsc[at];
          ks1 = s_ksc[at1];
          vs1 = s_vsc[at1];
        }
        if (nv >= 32)
          consume(s_kv[buf][team], ~0u, true, ks0, ks1, vs0, vs1);
        else
          consume(s_kv[buf][team], (1u << nv) - 1u, false, ks0, ks1, vs0, vs1);
      };
      u32x4 r0[PER], r1[PER];
      load(r0, 0);
      load(r1, 1);
      store(r0, 0, 0);
      load(r0, 2);
      __syncthreads();
      for (int u = 0; u < n_st; u += 2) {
        compute(u, 0);
        store(r1, u + 1, 1);
        load(r1, u + 3);
        __syncthreads();
        if (u + 1 >= n_st) break;  // uniform
        compute(u + 1, 1);
        store(r0, u + 2, 0);
        load(r0, u + 4);
        __syncthreads();
      }
    }

    // Drafts: rows of [node][d], V transposed on the way into LDS.
    for (int st = a > cache_stages ? a : cache_stages; st < z; ++st) {
      const int t0 = ((st - cache_stages) * SP + team) * 32;  // first node of the team's step
      __syncthreads();
      uint8_t* kv = s_kv[0][team];
      if (t0 < nodes) {
        for (int e = tt; e < 32 * (D / 8); e += TT) {
          const int t = e / (D / 8), ch = e - t * (D / 8);
          u32x4 kx{0u, 0u, 0u, 0u}, vx{0u, 0u, 0u, 0u};
          if (t0 + t < nodes) {
            const int64_t at = (((int64_t)b * p.num_nodes + t0 + t) * Hkv + g) * D + 8 * ch;
            kx = *(const u32x4*)(p.k_draft + at);
            vx = *(const u32x4*)(p.v_draft + at);
          }
          *(u32x4*)(kv + (ch * 32 + tree_row(t)) * 16) = kx;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *(uint16_t*)(kv + KB + tree_v_at(8 * ch + i, t >> 3) + 2 * (t & 7)) =
                (uint16_t)(vx[i >> 1] >> (16 * (i & 1)));
        }
      }
      __syncthreads();
      if (active && t0 < nodes)
        consume(kv, (uint32_t)(sees >> t0), false, p.scale_log2, p.scale_log2, 1.f, 1.f);
    }

    // The piece's result: teams merged in LDS, then the rows, or one partial.
    float l_tot = sum_xor32(l_run);
    if constexpr (SP > 1) {
      __syncthreads();
      if (h == 0) s_ml[wave][col] = make_float2(m_run, l_tot);
      __syncthreads();
      float M = kNoMax;
#pragma unroll
      for (int s = 0; s < SP; ++s) M = fmaxf(M, s_ml[s * NT + tile][col].x);
      l_tot = 0.f;
#pragma unroll
      for (int s = 0; s < SP; ++s) {
        const float2 ml = s_ml[s * NT + tile][col];
        l_tot += ml.y * (ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M));
      }
      const float f = m_run == M ? 1.f : __builtin_amdgcn_exp2f(m_run - M);
      m_run = M;
      f32x4* buf = (f32x4*)&s_kv[0][0][0];  // [team - 1][tile][4 * DB][64]
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 v{acc[i][4 * j] * f, acc[i][4 * j + 1] * f, acc[i][4 * j + 2] * f,
                        acc[i][4 * j + 3] * f};
          if (team > 0) {
            buf[(((team - 1) * NT + tile) * 4 * DB + 4 * i + j) * 64 + lane] = v;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][4 * j + e] = v[e];
          }
        }
      __syncthreads();
      if (team == 0) {
#pragma unroll
        for (int s = 0; s < SP - 1; ++s)
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x4 v = buf[((s * NT + tile) * 4 * DB + 4 * i + j) * 64 + lane];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][4 * j + e] += v[e];
            }
      }
    }
    const bool ends = z == sq.stages;
    if (a == 0 && ends) {
      if (team == 0 && mine) {
        const bool none = L == 0 && sees == 0;  // nothing to attend: zeros
        const float inv = none ? 0.f : 1.f / l_tot;
        uint16_t* o = p.out + row * D;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *(bf16x4*)(o + 32 * i + 8 * j + 4 * h) =
                bf16x4{(__bf16)(acc[i][4 * j] * inv), (__bf16)(acc[i][4 * j + 1] * inv),
                       (__bf16)(acc[i][4 * j + 2] * inv), (__bf16)(acc[i][4 * j + 3] * inv)};
      }
    } else {
      const int64_t slot = 2 * (int64_t)blockIdx.x + (first_piece ? 0 : 1);
      if (team == 0) {
        f32x4* po = (f32x4*)(p.part_o + (slot * NT + tile) * 32 * D);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            po[(4 * i + j) * 64 + lane] = f32x4{acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2],
                                                acc[i][4 * j + 3]};
        if (h == 0) p.part_ml[(slot * NT + tile) * 32 + col] = make_float2(m_run, l_tot);
      }
      if (a == 0 && tid == 0) {
        // pieces: this range's, and those of the ranges up to the segment's last stage
        const int last = x + sq.stages - 1;
        int w = (int)((int64_t)last * W / total);  // near the range that holds `last`
        while (w + 1 < W && (int64_t)total * (w + 1) / W <= last) ++w;
        while ((int64_t)total * w / W > last) --w;
        p.cuts[blockIdx.x] = make_int4(b, g * sq.blocks + blk, w - (int)blockIdx.x + 1, (int)slot);
      }
    }
    if (p.whole) return;
    x += z - a;
    if (x >= x1) return;  // uniform
    first_piece = false;
    while (s_pre[b + 1] <= x) ++b;
    b = uni(b);
  }
}

// Joins the pieces of the cut segment whose first piece workgroup blockIdx.x had: tile
// blockIdx.y.  Thread t holds accumulator quads t >> 6, (t >> 6) + 4, ... of lane t & 63.
template <int D, int NT>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeParams p) {
  constexpr int DB = D / 32, CB = 32 * NT;
  const int4 cut = p.cuts[blockIdx.x];
  if (cut.x < 0) return;
  const int b = cut.x, tile = blockIdx.y, lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
  const TreeSeq sq = tree_seq(p, b, 32, 1, CB);  // (only nodes, blocks and L > 0 matter here)
  const int g = cut.y / sq.blocks, blk = cut.y - g * sq.blocks;
  if (blk * CB + tile * 32 >= sq.nodes * p.group) return;  // no such columns
  float M = -__builtin_inff(), S = 0.f;
  f32x4 acc[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < cut.z; ++k) {
    const int64_t slot = k == 0 ? cut.w : 2 * ((int64_t)blockIdx.x + k);
    const float2 ml = p.part_ml[(slot * NT + tile) * 32 + col];
    const f32x4* po = (const f32x4*)(p.part_o + (slot * NT + tile) * 32 * D);
    f32x4 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = po[((threadIdx.x >> 6) + 4 * i) * 64 + lane];
    const float m = fmaxf(M, ml.x);
    const float f0 = M == m ? 1.f : __builtin_amdgcn_exp2f(M - m);
    const float f1 = ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - m);
    M = m;
    S = S * f0 + ml.y * f1;
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = acc[i] * f0 + o[i] * f1;
  }
  const int c = blk * CB + tile * 32 + col, node = c / p.group, head = c - node * p.group;
  if (node >= sq.nodes) return;
  const uint64_t live = sq.nodes >= 64 ? ~0ull : (1ull << sq.nodes) - 1;
  const bool none = sq.L == 0 && (p.tree_mask[(int64_t)b * p.num_nodes + node] & live) == 0;
  const float inv = none ? 0.f : 1.f / S;
  uint16_t* out = p.out + (((int64_t)b * p.num_nodes + node) * p.num_q_heads + g * p.group + head) * D;
#pragma unroll
  for (int k = 0; k < DB; ++k) {
    const int quad = (threadIdx.x >> 6) + 4 * k, i = quad >> 2, j = quad & 3;
    *(bf16x4*)(out + 32 * i + 8 * j + 4 * h) =
        bf16x4{(__bf16)(acc[k][0] * inv), (__bf16)(acc[k][1] * inv), (__bf16)(acc[k][2] * inv),
               (__bf16)(acc[k][3] * inv)};
  }
}

template <int D, int P, bool FP8>
static const void* tree_fn(int tiles) {
  return tiles == 1   ? (const void*)&tree_kernel<D, P, FP8, 1>
         : tiles == 2 ? (const void*)&tree_kernel<D, P, FP8, 2>
                      : (const void*)&tree_kernel<D, P, FP8, 4>;
}

int tree_workgroups_per_cu(int, int, bool, int tiles) { return tiles == 1 ? 1 : 2; }

hipError_t launch_tree(const TreeParams& p, int D, int P, bool fp8, int tiles, int64_t grid,
                       hipStream_t s) {
  const void* fn;
  if (D == 128)
    fn = P == 16 ? (fp8 ? tree_fn<128, 16, true>(tiles) : tree_fn<128, 16, false>(tiles))
                 : (fp8 ? tree_fn<128, 32, true>(tiles) : tree_fn<128, 32, false>(tiles));
  else
    fn = P == 16 ? (fp8 ? tree_fn<64, 16, true>(tiles) : tree_fn<64, 16, false>(tiles))
                 : (fp8 ? tree_fn<64, 32, true>(tiles) : tree_fn<64, 32, false>(tiles));
  TreeParams arg = p;
  void* args[] = {(void*)&arg};
  const unsigned lds = p.whole ? 0 : (unsigned)(p.num_seqs + 1) * 4;
  return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(64 * kTreeWaves), args, lds, s);
}

hipError_t launch_tree_combine(const TreeParams& p, int D, int tiles, int64_t grid, hipStream_t s) {
  const void* fn;
  if (D == 128)
    fn = tiles == 1   ? (const void*)&tree_combine_kernel<128, 1>
         : tiles == 2 ? (const void*)&tree_combine_kernel<128, 2>
                      : (const void*)&tree_combine_kernel<128, 4>;
  else
    fn = tiles == 1   ? (const void*)&tree_combine_kernel<64, 1>
         : tiles == 2 ? (const void*)&tree_combine_kernel<64, 2>
                      : (const void*)&tree_combine_kernel<64, 4>;
  TreeParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)grid, (unsigned)tiles), dim3(256), args, 0, s);
}

}  // namespace dora
