// Decode attention for a tree of drafted tokens per sequence, over the paged cache and the
// drafts' own keys and values.  All nodes of a sequence see its whole cache, so every
// cached byte is applied to the C = nodes x group columns of its KV head; among the drafts
// a column sees what its node's mask says.  This file: more than 32 columns, in blocks of 64 or
// 128, a tile of 32 for each of a workgroup's waves (fewer: tree_narrow.hip), and the
// join of cut segments.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tree_core.h"

namespace dora {

// Pages whose ids (and fp8 scales) a workgroup holds in LDS at a time.
constexpr int kTreeWindow = 512;

// Waits until at most N of the wave's loads are under way.
template <int N>
__device__ __forceinline__ void tree_wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
}

// 64 pieces of 16 bytes, one a lane, into LDS in lane order, past the registers.
__device__ __forceinline__ void tree_fetch(const uint8_t* from, uint8_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// A workgroup, a wave for each of its NT tiles of 32 columns, takes an equal, contiguous range of
// the batch's (sequence, KV head, column block, step) list, as the plain decode's wavefronts do,
// or, where p.whole, one (sequence, KV head, column block).
//   A step's pages go from HBM straight into one of three LDS buffers, as they are, two steps ahead
// of the one that all waves compute, with one barrier a step.  V's fp8 codes (K's too, but for CODES) are
// widened by each wave on the way into its products: four times the conversions of a kernel that
// does it on the way into LDS, but half the LDS traffic, and no registers or instructions for the
// way in (that one: 1,022 us for the 128-column fp8 rows below instead of 1,007, 156 for 139 in wide
// bf16 rows).  A fourth buffer: 1,000 and 140 us, but 137 for 124 in the 56-column rows.
//   Bound by no one unit: two waves a SIMD, whose vector and matrix instructions overlap in part.
// 256 fp8 rows of 4,096 tokens at the median, 16 nodes, 64/8 heads of 128 dims (128 columns): 3.3 GB
// and 0.80 TFLOP in 973 us with CODES, 0.82 PFLOP/s without the join of 25 us (a large bf16 product 1.34).  5 bf16 rows of 30,000, up to
// 64 nodes, 32/8 heads: 139 us, 0.5 PFLOP/s.  64 bf16 rows of 2,048 at the median, up to 8 nodes,
// 28/4 heads (56 columns): 0.50 GB in 124 us.  What does not pay: two tiles a wave straight from HBM
// (rows of 6,000 981 us instead of 1,010, of 500 1,440 instead of 960), registers for three waves
// a SIMD (they spill: wide rows 180), the next step's scores beside this one's weights.
template <int D, int P, bool FP8, int NT, bool CODES>
__global__ __launch_bounds__(64 * NT, 2) void tree_kernel(TreeParams p) {
  constexpr int TT = 64 * NT, PAIR = 32 / P, E = FP8 ? 1 : 2;
  constexpr int DB = D / 32, CB = 32 * NT;
  constexpr int TILE = P * D * E;         // bytes of one (page, KV head) tile
  constexpr int KB = PAIR * TILE;         // bytes of a step's K (V: as many)
  constexpr int NK = KB / 16;             // ... in pieces of 16
  constexpr int PER = 2 * NK / TT;        // pieces of a lane
  constexpr int ROW = P * E / 16;         // pieces of a V row of a page
  static_assert(2 * NK % TT == 0 && NK / PAIR % 64 == 0, "a wave's 64 pieces are on one page");
  typedef TreeRegs<D, P, FP8> R;
  typedef TreeTokens<P, FP8> Tok;
  // (three variables: the compiler waits for what is loaded into the one that is read)
  __shared__ __align__(16) uint8_t s_kv0[2 * KB], s_kv1[2 * KB], s_kv2[2 * KB];
  __shared__ int s_pid[kTreeWindow], s_odd[NT];
  __shared__ float s_ksc[FP8 ? kTreeWindow : 1], s_vsc[FP8 ? kTreeWindow : 1];
  extern __shared__ int s_pre[];

  const int tid = threadIdx.x, lane = tid & 63, tile = uni(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int Hkv = p.num_kv_heads, G = p.group;

  const int place = tree_place(p);
  TreeRange rg{0, 0, 0, 1, 0};
  int b;
  if (p.whole) {
    b = place / (Hkv * p.blocks);
  } else {
    rg = tree_range<P, 1, CB, kTreeWideCost, NT>(p, place, s_pre);
    if (tid == 0) p.cuts[place] = make_int4(-1, 0, 0, 0);
    if (rg.x0 >= rg.x1) return;  // uniform
    b = rg.b;
  }

  // In LDS a step's tiles are as in HBM, but that V's pieces of a row change places with the row,
  // so that 16 rows' pieces of one column lie in different banks.  v_lane: what lane's piece of V
  // is fetched from; k_at, v_turn: where the lane's operands are.
  auto turn_of = [](int d) { return ROW == 4 ? (d >> 2) & 3 : ROW == 2 ? (d >> 3) & 1 : 0; };
  const int v_lane = 16 * ((lane & ~(ROW - 1)) | ((lane & (ROW - 1)) ^ turn_of(lane / ROW)));
  const int ktok_ = Tok::of_row(col), v_turn = turn_of(col);
  const int k_at = (PAIR == 2 && ktok_ >= 16 ? TILE : 0) + (h * P + (ktok_ & (P - 1))) * 16;

  bool first_piece = true;
  int x = rg.x0;
  while (true) {
    // the piece: stages a .. z - 1 of (b, g, block)
    const TreeSeq sq = tree_seq(p, b, P, 1, CB);
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
    const int cache_stages = uni(sq.cache_stages);

    // queries: this lane's column (one that is not there takes node 0's, for nothing)
    const int c = blk * CB + tile * 32 + col;
    const int node = c / G, head = c - node * G;
    const bool mine = node < nodes;
    const int64_t row = (((int64_t)b * p.num_nodes + (mine ? node : 0)) * p.num_q_heads +
                         (int64_t)g * G + (mine ? head : 0));
    TreeQuery<D, FP8, CODES> qop;
    qop.load(p.q + row * D, h);
    const uint64_t live = nodes >= 64 ? ~0ull : (1ull << nodes) - 1;
    const uint64_t sees = mine ? p.tree_mask[(int64_t)b * p.num_nodes + node] & live : 0ull;
    const bool active = uni(blk * CB + tile * 32 < nodes * G);  // the wave's tile has columns

    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
    float m_run = kNoMax, l_run = 0.f;

    // Cached tokens, in windows of the pages whose ids fit the LDS array.
    constexpr int WST = kTreeWindow / PAIR;  // stages of a window
    const int c_end = z < cache_stages ? z : cache_stages;
    for (int w0 = a; w0 < c_end; w0 += WST) {
      const int n_st = c_end - w0 < WST ? c_end - w0 : WST;
      const int j0 = w0 * PAIR;
      const int n_win = n_pages - j0 < kTreeWindow ? n_pages - j0 : kTreeWindow;
      __syncthreads();  // the arrays and the buffers are free
      for (int t = tid; t < n_win; t += TT) {
        const int pid = p.block_table[(int64_t)b * p.stride + j0 + t];
        s_pid[t] = pid;
        if constexpr (FP8) {
          s_ksc[t] = p.k_scales[pid];
          s_vsc[t] = p.v_scales[pid];
        }
      }
      __syncthreads();
      // Pages of step w0 + u (past the end the window's last).
      auto page = [&](int u, int pg) {
        const int at = u * PAIR + pg;
        return s_pid[at < n_win ? at : n_win - 1];
      };
      auto fetch = [&](uint8_t* kv, int u, int v0, int v1) {
        const bool past = u >= n_st;  // past the end the loads still issue, one line each
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
          tree_fetch(at + (past ? 0 : is_v ? v_lane : 16 * lane), kv + e0 * 16);
        }
      };
      auto compute = [&](const uint8_t* kv, int u) {
        if (!active || u >= n_st) return;  // uniform in the wave
        const int nv = L - (w0 + u) * 32;
        float ks0 = 1.f, ks1 = 1.f, vs0 = 1.f, vs1 = 1.f;
        if constexpr (FP8) {
          const int at = u * PAIR, at1 = PAIR == 2 && at + 1 < n_win ? at + 1 : at;
          ks0 = s_ksc[at];
          vs0 = s_vsc[at];
          ks1 = s_ksc[at1];
          vs1 = s_vsc[at1];
        }
        const TreeScale s0 = tree_scale<FP8>(p.scale_log2, ks0, vs0);
        const TreeScale s1 = PAIR == 2 ? tree_scale<FP8>(p.scale_log2, ks1, vs1) : s0;
        const bool masked = nv < 32;
        const uint32_t own = masked ? Tok::registers((1u << nv) - 1u, h) : 0xFFFFu;
        R r;
#pragma unroll
        for (int s = 0; s < R::NK; ++s) r.k[s] = *(const u32x4*)(kv + k_at + s * (2 * P * 16));
        __builtin_amdgcn_sched_barrier(0);
        tree_step<D, FP8>(
            [&] { return tree_scores(r, qop); },
            [&] {  // V is read behind the scores, and waited for behind the softmax
              typedef typename R::vraw_t V;
#pragma unroll
              for (int i = 0; i < DB; ++i) {
                const uint8_t* row_ = kv + KB + (32 * i + col) * ROW * 16;
                if constexpr (R::RUN16) {
                  r.v[i] = *(const V*)(row_ + 16 * (h ^ v_turn));
                } else {
#pragma unroll
                  for (int s = 0; s < 2; ++s) {
                    if constexpr (FP8)
                      r.v[2 * i + s] = *(const V*)(row_ + s * TILE + 8 * h);
                    else if constexpr (PAIR == 2)
                      r.v[2 * i + s] = *(const V*)(row_ + s * TILE + 16 * (h ^ v_turn));
                    else
                      r.v[2 * i + s] = *(const V*)(row_ + 16 * ((2 * s + h) ^ v_turn));
                  }
                }
              }
              __builtin_amdgcn_sched_barrier(0);
              if (masked) tree_keep(r, own);  // slots past the sequence hold anything
            },
            [&](int i, int s) { return tree_v(r, i, s); }, s0, s1, masked, own, acc, m_run, l_run);
      };
      // Two stages on their way into LDS while a third is computed.  A wave's part of stage u has
      // arrived when only the next stage's is under way, and all waves' when they have met;
      // then they are done with stage u - 1 too, whose buffer takes stage u + 2.
      int v0 = page(1, 0), v1 = page(1, 1);
      fetch(s_kv0, 0, page(0, 0), page(0, 1));
      fetch(s_kv1, 1, v0, v1);
      v0 = page(2, 0);
      v1 = page(2, 1);
      auto turn = [&](uint8_t* now, uint8_t* next, int u) {
        tree_wait_loads<PER>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        fetch(next, u + 2, v0, v1);
        v0 = page(u + 3, 0);
        v1 = page(u + 3, 1);
        compute(now, u);
        __builtin_amdgcn_sched_barrier(0);
      };
      for (int u = 0; u < n_st; u += 3) {
        turn(s_kv0, s_kv2, u);
        turn(s_kv1, s_kv0, u + 1);
        turn(s_kv2, s_kv1, u + 2);
      }
      tree_wait_loads<0>();  // (the buffers are written otherwise below)
    }

    // Drafts (the last stages).  V is turned round on the way into LDS.
    int any_odd = 0;  // among V something is not finite
    for (int st = a > cache_stages ? a : cache_stages; st < z; ++st) {
      const int t0 = (st - cache_stages) * 32;  // first node of the step
      __syncthreads();
      uint8_t* vt = s_kv0;  // [d][32 nodes]
      const bool odd = tree_put_drafts<D, TT>(p, vt, b, g, t0, nodes, tid);
      if (lane == 0) s_odd[tile] = odd;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NT; ++w) any_odd |= s_odd[w];  // (stored again behind the next step's first barrier)
      if (!active) continue;  // uniform in the wave
      const int ktok = Tok::of_row(col);
      const int t = t0 + ktok < nodes ? t0 + ktok : nodes - 1;  // a row past the nodes is masked
      const uint16_t* kd = p.k_draft + (((int64_t)b * p.num_nodes + t) * Hkv + g) * D;
      const TreeScale one{p.scale_log2, 0.f, 1.f, 1.f};
      tree_step<D, FP8>(
          [&] { return tree_draft_scores(kd, p.q + row * D, qop, h); },
          [] {},
          [&](int i, int s) {
            return *(const bf16x8*)(vt + tree_v_at(32 * i + col, Tok::RUN16 ? 2 * h + s : 2 * s + h));
          },
          one, one, true, Tok::registers((uint32_t)(sees >> t0), h), acc, m_run, l_run);
    }

    // The piece's result: rows, or one partial.
    const float S = sum_xor32(l_run);
    const bool whole = a == 0 && z == sq.stages;
    const int64_t slot = 2 * (int64_t)place + (first_piece ? 0 : 1);
    const bool none = L == 0 && sees == 0;  // nothing to attend: zeros
    const float inv = none ? 0.f : 1.f / S;
#pragma unroll
    for (int quad = 0; quad < 4 * DB; ++quad) {
      const int i = quad >> 2, j = quad & 3;
      const f32x4 o{acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]};
      if (!whole) {
        if (active) ((f32x4*)(p.part_o + (slot * NT + tile) * 32 * D))[quad * 64 + lane] = o;
      } else if (mine) {
        *(bf16x4*)(p.out + row * D + 32 * i + 8 * j + 4 * h) =
            bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv),
                   (__bf16)(o[3] * inv)};
      }
    }
    if (__builtin_expect(uni(any_odd) && active, 0)) {
      // the piece's own drafts, one step's or both: another's may weigh nothing in this piece
      const uint64_t own = (a > cache_stages ? ~0ull << 32 : ~0ull) & (z > cache_stages + 1 ? ~0ull : ~0u);
      for (int quad = 0; quad < 4 * DB; ++quad) {
        const int d0 = tree_quad_dim(quad, h);
        const f32x4 add = tree_odd_values(p, D, b, g, sees & own, d0);
        if (!whole)
          tree_add_odd(&((f32x4*)(p.part_o + (slot * NT + tile) * 32 * D))[quad * 64 + lane], add);
        else if (mine)
          tree_add_odd((bf16x4*)(p.out + row * D + d0), add);
      }
    }
    if (!whole && active && h == 0)
      p.part_ml[(slot * NT + tile) * 32 + col] = make_float2(m_run, S);
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

// CODES where vector instructions bound the waves (four tiles) and rows may be long enough for the
// queries' codes, about 1 us a segment.  128 columns, fp8, against the widened codes: rows of 6,000 tokens
// (256) 962 us for 1,024 (128 dims, pages of 32), 1,014 for 1,061 (16), 64 dims 626 for 658 and 690 for
// 706; rows of 1,500 (800) and 700 (1,600) level; in two tiles or whole rows of 500 slower by 4 to 5%.
template <int D, int P, bool FP8>
static const void* wide_fn(int tiles, bool whole) {
  if constexpr (FP8)
    if (tiles == 4 && !whole) return (const void*)&tree_kernel<D, P, true, 4, true>;
  return tiles == 2 ? (const void*)&tree_kernel<D, P, FP8, 2, false>
                    : (const void*)&tree_kernel<D, P, FP8, 4, false>;
}

hipError_t launch_tree_wide(const TreeParams& p, int D, int P, bool fp8, int tiles, int64_t grid,
                            hipStream_t s) {
  const void* fn;
  if (D == 128)
    fn = P == 16 ? (fp8 ? wide_fn<128, 16, true>(tiles, p.whole) : wide_fn<128, 16, false>(tiles, p.whole))
                 : (fp8 ? wide_fn<128, 32, true>(tiles, p.whole) : wide_fn<128, 32, false>(tiles, p.whole));
  else
    fn = P == 16 ? (fp8 ? wide_fn<64, 16, true>(tiles, p.whole) : wide_fn<64, 16, false>(tiles, p.whole))
                 : (fp8 ? wide_fn<64, 32, true>(tiles, p.whole) : wide_fn<64, 32, false>(tiles, p.whole));
  TreeParams arg = p;
  void* args[] = {(void*)&arg};
  const unsigned lds = p.whole ? 0 : (unsigned)(p.num_seqs + 1) * 4;
  return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(64 * tiles), args, lds, s);
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
  return hipLaunchKernel(fn, dim3((unsigned)grid, (unsigned)tiles, (unsigned)(D / 32)), dim3(256), args, 0, s);
}

}  // namespace dora
