// Decode attention for a tree of drafted tokens per sequence, over the paged cache and the
// drafts' own keys and values.  All nodes of a sequence see its whole cache, so every
// cached byte is applied to the C = nodes x group columns of its KV head; among the drafts
// a column sees what its node's mask says.  This file: more than 64 columns, in blocks of
// 128, a tile of 32 for each of a workgroup's four waves (fewer: tree_narrow.hip), and the
// join of cut segments.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tree_core.h"

namespace dora {

constexpr int kTreeTiles = kTreeWaves;  // of a column block, at most
// Pages whose ids (and fp8 scales) a workgroup holds in LDS at a time.
constexpr int kTreeWindow = 512;
// What a segment costs besides its steps (lengths, page ids, queries, the rows), in steps; 256
// fp8 rows of 2,048 tokens at the median, 8 nodes: 539 us against 633 at 0.
constexpr int kTreeWideCost = 4;

// Row of a 32-token tile that holds token t, and the other way round (bits 2 and 3
// change places): the rows of a lane's accumulator, 16s + 8j + 4h + i, then are the tokens
// 16s + 8h + 4j + i, the 8 consecutive tokens of k-step s that this lane supplies to the
// second product.
__device__ __forceinline__ int tree_row(int t) {
  return (t & 0x13) | ((t & 4) << 1) | ((t & 8) >> 1);
}
// Registers of half h whose tokens are among `bits`.
__device__ __forceinline__ uint32_t tree_registers(uint32_t bits, int h) {
  return ((bits >> (8 * h)) & 0xFFu) | (((bits >> (16 + 8 * h)) & 0xFFu) << 8);
}

// V's 16-byte pieces (8 tokens of a head-dim row, 4 pieces a row) change places with
// the row so that 16 rows' pieces of one column lie in different banks.
__device__ __forceinline__ int tree_v_at(int row, int piece) {
  return row * 64 + ((piece ^ ((row >> 2) & 3)) << 4);
}

// A workgroup takes an equal, contiguous range of the batch's (sequence, KV head, column
// block, step) list, as the plain decode's wavefronts do, or, where p.whole, one
// (sequence, KV head, column block).
//   A step's pages go HBM -> registers (two steps in flight; teams of two waves, whose shares
// are twice as large, one: 122 us against 139 for the bf16 rows below) -> LDS, fp8 widened to bf16
// on the way, so that the four waves share one read and one conversion.
//   Bound by no one unit: with two waves a SIMD, the matrix pipe is busy for 41% of the cycles,
// the vector ALU for 59% (16 of its 80 instructions a step are exponentials of 16 cycles), LDS
// for 60%.  256 fp8 rows of 4,096 tokens at the median, 16 nodes, 64/8 heads of 128 dims (128
// columns): 3.3 GB and 0.80 TFLOP in 1,040 us, 0.77 PFLOP/s (a large bf16 product 1.34).  64
// bf16 rows of 2,048 at the median, up to 8 nodes, 28/4 heads (56 columns): 0.50 GB in 122 us.
// Two tiles a wave without LDS for K and V (981 us for rows of 6,000 instead of 1,010, 1,440 for
// rows of 500 instead of 960), a third workgroup per CU (bf16 145 -> 178 us) and the next step's
// scores beside this one's weights (1,035 -> 1,107) do not pay.
template <int D, int P, bool FP8, int NT>
__global__ __launch_bounds__(64 * kTreeWaves, 2) void tree_kernel(TreeParams p) {
  constexpr int SP = kTreeWaves / NT, TT = 64 * NT, PAIR = 32 / P;
  constexpr int KS = D / 16, DB = D / 32, CB = 32 * NT;
  constexpr int DEPTH = NT == 2 ? 1 : 2;
  constexpr int TILE = P * D * (FP8 ? 1 : 2);      // bytes of one (page, KV head) tile
  constexpr int NK = 32 * D * (FP8 ? 1 : 2) / 16;  // 16-byte pieces of a step's K (V: as many)
  constexpr int PER = 2 * NK / TT;                 // pieces of a thread
  constexpr int KB = 32 * D * 2;                   // LDS bytes of a step's K (V: as many)
  static_assert(2 * NK % TT == 0 && NK / PAIR % 64 == 0, "a wave's 64 pieces are on one page");
  __shared__ __align__(16) uint8_t s_kv[2][SP][2 * KB];
  __shared__ int s_pid[kTreeWindow];
  __shared__ float s_ksc[FP8 ? kTreeWindow : 1], s_vsc[FP8 ? kTreeWindow : 1];
  __shared__ float2 s_ml[kTreeWaves][32];
  extern __shared__ int s_pre[];

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int team = wave / NT, tile = wave % NT, tt = tid - team * TT;
  const int Hkv = p.num_kv_heads, G = p.group;

  const int place = tree_place(p);
  TreeRange rg{0, 0, 0, 1, 0};
  int b;
  if (p.whole) {
    b = place / (Hkv * p.blocks);
  } else {
    rg = tree_range<P, SP, CB, kTreeWideCost>(p, place, s_pre);
    if (tid == 0) p.cuts[place] = make_int4(-1, 0, 0, 0);
    if (rg.x0 >= rg.x1) return;  // uniform
    b = rg.b;
  }

  bool first_piece = true;
  int x = rg.x0;
  while (true) {
    // the piece: stages a .. z - 1 of (b, g, block)
    const TreeSeq sq = tree_seq(p, b, P, SP, CB);
    int g, blk, a, z, taken = 0;
    if (p.whole) {
      const int r = place - b * Hkv * p.blocks;
      g = r / p.blocks;
      blk = r - g * p.blocks;
      a = 0;
      z = sq.stages;
      if (blk >= sq.blocks) return;  // uniform: no such columns (or no nodes)
    } else {
      const int r = x - s_pre[b], len = sq.stages + kTreeWideCost;
      const int gb = r / len;
      g = gb / sq.blocks;
      blk = gb - g * sq.blocks;
      a = r - gb * len;
      z = len - a < rg.x1 - x ? len : a + (rg.x1 - x);
      taken = z - a;
      a = a > kTreeWideCost ? a - kTreeWideCost : 0;
      z -= kTreeWideCost;
    }
    if (z <= a) {  // uniform: nothing but a start, which is the next workgroup's
      x += taken;
      if (x >= rg.x1) return;
      continue;
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

    // The step in buffer `buf`; masked: the tokens of `bits` alone count.
    auto consume = [&](int buf, bool masked, uint32_t bits, const TreeScale& s0, const TreeScale& s1) {
      const uint8_t* kv = s_kv[buf][team];
      const uint32_t own = masked ? tree_registers(bits, h) : 0xFFFFu;
      tree_step<D, FP8, NT == 4>(
          [&](int s) { return *(const bf16x8*)(kv + ((2 * s + h) * 32 + col) * 16); },
          [&](int i, int s) { return *(const bf16x8*)(kv + KB + tree_v_at(32 * i + col, 2 * s + h)); },
          s0, s1, masked, own, qop, acc, m_run, l_run);
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
          s_ksc[t] = p.k_scales[pid];
          s_vsc[t] = p.v_scales[pid];
        }
      }
      __syncthreads();
      // Pages of the team's step of stage w0 + u (past the end the window's last).
      auto page = [&](int u, int pg) {
        const int at = (u * SP + team) * PAIR + pg;
        return s_pid[at < n_win ? at : n_win - 1];
      };
      auto load = [&](u32x4 (&r)[PER], int u, int v0, int v1) {
        const int each = u < n_st ? 16 : 0;  // past the end the loads still issue, one line each
        const int p0 = uni(v0), p1 = uni(v1);
        const int64_t base0 = (int64_t)p0 * p.page_bytes + (int64_t)g * TILE;
        const int64_t base1 = (int64_t)p1 * p.page_bytes + (int64_t)g * TILE;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int e0 = 64 * tile + TT * k;  // the wave's first piece
          const bool is_v = NK % TT == 0 ? TT * k >= NK : e0 >= NK;
          const int i0 = is_v ? e0 - NK : e0;
          const bool second = PAIR == 2 && i0 >= NK / 2;
          const int rem = (second ? i0 - NK / 2 : i0) * 16;
          const uint8_t* at = (is_v ? p.v_pages : p.k_pages) + (second ? base1 : base0) + rem;
          r[k] = __builtin_nontemporal_load((const u32x4*)(at + lane * each));
        }
      };
      auto store = [&](const u32x4 (&r)[PER], int u, int buf) {
        uint8_t* kv = s_kv[buf][team];
        const int nv = L - ((w0 + u) * SP + team) * 32;  // tokens of the step that count
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int e = tt + k * TT;
          const bool is_v = NK % TT == 0 ? TT * k >= NK : 64 * tile + TT * k >= NK;
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
            if (nv < 32) {  // uniform: slots past the sequence hold anything
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
        if (!active || u >= n_st || step >= cache_steps) return;  // uniform in the wave
        const int nv = L - step * 32;
        float ks0 = 1.f, ks1 = 1.f, vs0 = 1.f, vs1 = 1.f;
        if constexpr (FP8) {
          const int at = (u * SP + team) * PAIR, at1 = PAIR == 2 && at + 1 < n_win ? at + 1 : at;
          ks0 = s_ksc[at];
          vs0 = s_vsc[at];
          ks1 = s_ksc[at1];
          vs1 = s_vsc[at1];
        }
        const TreeScale s0 = tree_scale<FP8>(p.scale_log2, ks0, vs0);
        const TreeScale s1 = PAIR == 2 ? tree_scale<FP8>(p.scale_log2, ks1, vs1) : s0;
        consume(buf, nv < 32, nv < 32 ? (1u << nv) - 1u : ~0u, s0, s1);
      };
      if constexpr (DEPTH == 1) {
        // One stage in flight in registers, two in LDS: stage u + 1 goes from registers to
        // LDS, and the loads of stage u + 2 are issued, before stage u is computed.
        u32x4 r0[PER];
        load(r0, 0, page(0, 0), page(0, 1));
        int v0 = page(1, 0), v1 = page(1, 1);
        store(r0, 0, 0);
        load(r0, 1, v0, v1);
        for (int u = 0; u < n_st; ++u) {
          __syncthreads();
          v0 = page(u + 2, 0);
          v1 = page(u + 2, 1);
          store(r0, u + 1, (u + 1) & 1);
          load(r0, u + 2, v0, v1);
          compute(u, u & 1);
        }
      } else {
        u32x4 r0[PER], r1[PER];
        int v0 = page(1, 0), v1 = page(1, 1);
        load(r0, 0, page(0, 0), page(0, 1));
        load(r1, 1, v0, v1);
        v0 = page(2, 0);
        v1 = page(2, 1);
        store(r0, 0, 0);
        load(r0, 2, v0, v1);
        for (int u = 0; u < n_st; u += 2) {
          __syncthreads();
          v0 = page(u + 3, 0);
          v1 = page(u + 3, 1);
          store(r1, u + 1, 1);
          load(r1, u + 3, v0, v1);
          compute(u, 0);
          // (no way out here: the compiler would wait at the top for what is loaded below)
          __syncthreads();
          v0 = page(u + 4, 0);
          v1 = page(u + 4, 1);
          store(r0, u + 2, 0);
          load(r0, u + 4, v0, v1);
          compute(u + 1, 1);
        }
      }
    }

    // Drafts: rows of [node][d], V turned round on the way into LDS.
    for (int st = a > cache_stages ? a : cache_stages; st < z; ++st) {
      const int t0 = ((st - cache_stages) * SP + team) * 32;  // first node of the team's step
      __syncthreads();
      uint8_t* kv = s_kv[0][team];
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
      __syncthreads();
      const TreeScale one{p.scale_log2, 0.f, 1.f, 1.f};
      if (active && t0 < nodes) consume(0, true, (uint32_t)(sees >> t0), one, one);
    }

    // The piece's result: a tile's SP waves merged in LDS, each summing a share of the quads;
    // then the rows, or one partial.
    constexpr int QUADS = 4 * DB;
    float S = sum_xor32(l_run), M = m_run;
    f32x4* s_o = (f32x4*)&s_kv[0][0][0];  // [wave][quad][lane]
    if constexpr (SP > 1) {
      __syncthreads();  // the buffers are free
      if (h == 0) s_ml[wave][col] = make_float2(m_run, S);
      __syncthreads();
#pragma unroll
      for (int w = 0; w < SP; ++w) M = fmaxf(M, s_ml[w * NT + tile][col].x);
      S = 0.f;
#pragma unroll
      for (int w = 0; w < SP; ++w) {
        const float2 ml = s_ml[w * NT + tile][col];
        S += ml.y * (ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M));
      }
      const float f = m_run == M ? 1.f : __builtin_amdgcn_exp2f(m_run - M);
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s_o[(wave * QUADS + 4 * i + j) * 64 + lane] =
              f32x4{acc[i][4 * j] * f, acc[i][4 * j + 1] * f, acc[i][4 * j + 2] * f,
                    acc[i][4 * j + 3] * f};
      __syncthreads();
    }
    const bool whole = a == 0 && z == sq.stages;
    const int64_t slot = 2 * (int64_t)place + (first_piece ? 0 : 1);
    const bool none = L == 0 && sees == 0;  // nothing to attend: zeros
    const float inv = none ? 0.f : 1.f / S;
#pragma unroll
    for (int k = 0; k < QUADS / SP; ++k) {
      const int quad = team + SP * k, i = quad >> 2, j = quad & 3;
      f32x4 o;
      if constexpr (SP > 1) {
        o = s_o[(tile * QUADS + quad) * 64 + lane];
#pragma unroll
        for (int w = 1; w < SP; ++w) o += s_o[((w * NT + tile) * QUADS + quad) * 64 + lane];
      } else {
        o = f32x4{acc[k >> 2][4 * (k & 3)], acc[k >> 2][4 * (k & 3) + 1], acc[k >> 2][4 * (k & 3) + 2],
                  acc[k >> 2][4 * (k & 3) + 3]};
      }
      if (!whole) {
        if (active) ((f32x4*)(p.part_o + (slot * NT + tile) * 32 * D))[quad * 64 + lane] = o;
      } else if (mine) {
        *(bf16x4*)(p.out + row * D + 32 * i + 8 * j + 4 * h) =
            bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv),
                   (__bf16)(o[3] * inv)};
      }
    }
    if (!whole && active && team == 0 && h == 0)
      p.part_ml[(slot * NT + tile) * 32 + col] = make_float2(M, S);
    if (!whole && a == 0 && tid == 0)
      p.cuts[place] = make_int4(b, g * sq.blocks + blk,
                                     tree_pieces(rg, place, x + taken + (sq.stages - z) - 1), (int)slot);
    if (p.whole) return;
    x += taken;
    if (x >= rg.x1) return;  // uniform
    first_piece = false;
    while (s_pre[b + 1] <= x) ++b;
    b = uni(b);
  }
}

// Joins the pieces of the cut segment whose first piece the workgroup of this place had: tile
// blockIdx.y, accumulator quads 4 blockIdx.z .. + 3 (rows 32 blockIdx.z .. + 31 of the head's
// dim), one a wave.  A read of the partials, little else: many small workgroups, and the
// loads of kTreeJoin pieces at a time.
constexpr int kTreeJoin = 4;
template <int D, int NT>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeParams p) {
  constexpr int CB = 32 * NT;
  const int place = tree_place(p);
  const int4 cut = p.cuts[place];
  if (cut.x < 0) return;
  const int b = cut.x, tile = blockIdx.y, lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
  const TreeSeq sq = tree_seq(p, b, 32, 1, CB);  // (only nodes, blocks and L > 0 matter here)
  const int j = threadIdx.x >> 6, quad = 4 * blockIdx.z + j;
  float M = -__builtin_inff(), S = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f}, o[kTreeJoin];
  float2 ml[kTreeJoin];
  auto load = [&](int k0) {
#pragma unroll
    for (int k = 0; k < kTreeJoin; ++k) {  // past the end the last piece's again
      const int at = k0 + k < cut.z ? k0 + k : cut.z - 1;
      const int64_t slot = at == 0 ? cut.w : 2 * ((int64_t)place + at);
      ml[k] = p.part_ml[(slot * NT + tile) * 32 + col];
      o[k] = ((const f32x4*)(p.part_o + (slot * NT + tile) * 32 * D))[quad * 64 + lane];
    }
  };
  load(0);  // beside the sequence's lengths
  __builtin_amdgcn_sched_barrier(0);
  const int g = cut.y / sq.blocks, blk = cut.y - g * sq.blocks;
  const int c = blk * CB + tile * 32 + col, node = c / p.group, head = c - node * p.group;
  if (blk * CB + tile * 32 >= sq.nodes * p.group) return;  // no such columns
  const uint64_t live = sq.nodes >= 64 ? ~0ull : (1ull << sq.nodes) - 1;
  const bool mine = node < sq.nodes;
  const bool none = sq.L == 0 && mine && (p.tree_mask[(int64_t)b * p.num_nodes + node] & live) == 0;
  for (int k0 = 0; k0 < cut.z; k0 += kTreeJoin) {
    if (k0 > 0) load(k0);
    float m = M;
#pragma unroll
    for (int k = 0; k < kTreeJoin; ++k) m = fmaxf(m, ml[k].x);
    const float f0 = M == m ? 1.f : __builtin_amdgcn_exp2f(M - m);
    M = m;
    S *= f0;
    acc *= f0;
#pragma unroll
    for (int k = 0; k < kTreeJoin; ++k) {
      if (k0 + k >= cut.z) break;  // uniform
      const float f = ml[k].x == m ? 1.f : __builtin_amdgcn_exp2f(ml[k].x - m);
      S += ml[k].y * f;
      acc += o[k] * f;
    }
  }
  if (!mine) return;
  const float inv = none ? 0.f : 1.f / S;
  uint16_t* out = p.out + (((int64_t)b * p.num_nodes + node) * p.num_q_heads + g * p.group + head) * D;
  *(bf16x4*)(out + 32 * blockIdx.z + 8 * j + 4 * h) =
      bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
             (__bf16)(acc[3] * inv)};
}

template <int D, int P, bool FP8>
static const void* wide_fn(int tiles) {
  return tiles == 2 ? (const void*)&tree_kernel<D, P, FP8, 2>
                    : (const void*)&tree_kernel<D, P, FP8, kTreeTiles>;
}

hipError_t launch_tree_wide(const TreeParams& p, int D, int P, bool fp8, int tiles, int64_t grid,
                            hipStream_t s) {
  const void* fn;
  if (D == 128)
    fn = P == 16 ? (fp8 ? wide_fn<128, 16, true>(tiles) : wide_fn<128, 16, false>(tiles))
                 : (fp8 ? wide_fn<128, 32, true>(tiles) : wide_fn<128, 32, false>(tiles));
  else
    fn = P == 16 ? (fp8 ? wide_fn<64, 16, true>(tiles) : wide_fn<64, 16, false>(tiles))
                 : (fp8 ? wide_fn<64, 32, true>(tiles) : wide_fn<64, 32, false>(tiles));
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
                      : (const void*)&tree_combine_kernel<128, kTreeTiles>;
  else
    fn = tiles == 1   ? (const void*)&tree_combine_kernel<64, 1>
         : tiles == 2 ? (const void*)&tree_combine_kernel<64, 2>
                      : (const void*)&tree_combine_kernel<64, kTreeTiles>;
  TreeParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)grid, (unsigned)tiles, (unsigned)(D / 32)), dim3(256), args, 0, s);
}

}  // namespace dora
