// Tree attention for at most 32 columns (nodes x group) per KV head, a tile: the waves of a
// workgroup take its steps in turn, and load them straight from HBM into matrix operands.
// Bound by memory: 64 bf16 rows of 2,048 tokens at the median, 4 nodes, 28/4 heads of 128 dims:
// 0.48 GB in 92 us with the join, 5.2 TB/s (through LDS, as tree.hip: 114); 256 fp8 rows, 64/8
// heads, 2.0 GB in 369 us, 5.3 TB/s (431).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tree_core.h"

namespace dora {

template <int D, int P, bool FP8>
__global__ __launch_bounds__(64 * kTreeWaves, FP8 || D == 64 ? 2 : 1) void tree_narrow_kernel(TreeParams p) {
  constexpr int SP = kTreeWaves, PAIR = 32 / P;
  constexpr int DB = D / 32, E = FP8 ? 1 : 2;
  constexpr int TILE = P * D * E;  // bytes of one (page, KV head) tile
  constexpr int QUADS = 4 * DB;    // accumulator quads of a tile
  typedef TreeRegs<D, P, FP8> R;
  typedef TreeTokens<P, FP8> Tok;
  __shared__ __align__(16) f32x4 s_o[kTreeWaves][QUADS][64];  // merge; a wave's draft V before
  __shared__ float2 s_ml[kTreeWaves][32];
  __shared__ int s_odd[kTreeWaves];
  extern __shared__ int s_pre[];

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int Hkv = p.num_kv_heads, G = p.group;

  const int place = tree_place(p);
  TreeRange rg{0, 0, 0, 1, 0};
  int b;
  if (p.whole) {
    b = place / Hkv;
  } else {
    rg = tree_range<P, SP, 32, kTreeNarrowCost, SP>(p, place, s_pre);
    if (tid == 0) p.cuts[place] = make_int4(-1, 0, 0, 0);
    if (rg.x0 >= rg.x1) return;  // uniform
    b = rg.b;
  }

  // Per-lane byte offsets inside a (page, KV head) tile, and which of a step's two pages
  // the lane's K token is on.
  const int ktok = Tok::of_row(col);
  const uint32_t koff = (uint32_t)((h * P + (ktok & (P - 1))) * 16);
  const bool ksecond = PAIR == 2 && ktok >= 16;
  const uint32_t voff = (uint32_t)(col * P * E + (Tok::RUN16 ? 16 * h : 8 * h * E));

  bool first_piece = true;
  int x = rg.x0;
  while (true) {
    // the piece: stages a .. z - 1 of (b, g)
    const TreeSeq sq = tree_seq(p, b, P, SP, 32);
    int g, a, z, taken = 0;
    if (p.whole) {
      g = place - b * Hkv;
      a = 0;
      z = sq.stages;
      if (sq.nodes == 0) return;  // uniform
    } else {
      const int r = x - s_pre[b], len = sq.stages + kTreeNarrowCost;
      g = r / len;
      a = r - g * len;
      z = len - a < rg.x1 - x ? len : a + (rg.x1 - x);
      taken = z - a;
      a = a > kTreeNarrowCost ? a - kTreeNarrowCost : 0;
      z -= kTreeNarrowCost;
    }
    if (z <= a) {  // uniform: nothing but a start, which is the next workgroup's
      x += taken;
      if (x >= rg.x1) return;
      continue;
    }
    g = uni(g);
    a = uni(a);
    z = uni(z);
    const int L = uni(sq.L), nodes = uni(sq.nodes), n_pages = uni(sq.pages);
    const int cache_steps = uni(sq.cache_steps), cache_stages = uni(sq.cache_stages);

    // this wave's steps of the cache: st0, st0 + SP, ...; lane u holds the pages of its u-th
    const int st0 = a * SP + wave;
    const int c_end = z < cache_stages ? z * SP : cache_steps;  // past the piece's last step
    int steps = c_end > st0 ? (c_end - st0 + SP - 1) / SP : 0;
    const int32_t* row_ids = p.block_table + (int64_t)b * p.stride;
    int pid0 = 0, pid1 = 0;
    auto load_ids = [&](int u0) {  // of the wave's steps u0 .. u0 + 63
      const int j = (st0 + SP * (u0 + lane)) * PAIR;
      const int last = n_pages - 1;
      pid0 = row_ids[j < last ? j : last];
      if constexpr (PAIR == 2) pid1 = row_ids[j + 1 < last ? j + 1 : last];
    };
    if (steps > 0) load_ids(0);

    // queries and mask: this lane's column (one that is not there takes node 0's, for nothing)
    const int node = col / G, head = col - node * G;
    const bool mine = node < nodes;
    const int64_t row = (((int64_t)b * p.num_nodes + (mine ? node : 0)) * p.num_q_heads +
                         (int64_t)g * G + (mine ? head : 0));
    TreeQuery<D, FP8, false> qop;
    qop.load(p.q + row * D, h);
    uint64_t sees = p.tree_mask[(int64_t)b * p.num_nodes + (mine ? node : 0)];
    sees &= nodes >= 64 ? ~0ull : (1ull << nodes) - 1;
    if (!mine) sees = 0;

    f32x16 acc[DB];
    float m_run = kNoMax, l_run = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    // Cached tokens, 64 steps of the wave at a time (as many as lanes hold pages of).
    for (int u0 = 0; u0 < steps; u0 += 64) {
      if (u0 > 0) load_ids(u0);
      const int n = steps - u0 < 64 ? steps - u0 : 64;
      R buf[2];
      float ks0[2], ks1[2], vs0[2], vs1[2];
      auto prefetch = [&](int r, int u) {
        const bool past = u >= n;  // past the last step the loads still issue, one line each
        u = past ? n - 1 : u;
        const int p0 = __builtin_amdgcn_readlane(pid0, u);
        const int p1 = PAIR == 2 ? __builtin_amdgcn_readlane(pid1, u) : p0;
        if constexpr (FP8) {
          ks0[r] = p.k_scales[p0];
          vs0[r] = p.v_scales[p0];
          ks1[r] = PAIR == 2 ? p.k_scales[p1] : ks0[r];
          vs1[r] = PAIR == 2 ? p.v_scales[p1] : vs0[r];
        }
        const int64_t base0 = (int64_t)p0 * p.page_bytes + (int64_t)g * TILE;
        const int64_t base1 = (int64_t)p1 * p.page_bytes + (int64_t)g * TILE;
        const uint8_t* kb = p.k_pages + (ksecond ? base1 : base0) + (past ? 0u : koff);
#pragma unroll
        for (int s = 0; s < R::NK; ++s)
          buf[r].k[s] = tree_load<u32x4>(kb + s * (2 * P * 16));
        const uint8_t* vb0 = p.v_pages + base0 + (past ? 0u : voff);
        const uint8_t* vb1 = p.v_pages + base1 + (past ? 0u : voff);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          typedef typename R::vraw_t V;
          constexpr int BLK = 32 * P * E;  // bytes between 32-row blocks
          if constexpr (R::RUN16) {
            buf[r].v[i] = tree_load<V>(vb0 + i * BLK);
          } else if constexpr (PAIR == 2) {
            buf[r].v[2 * i] = tree_load<V>(vb0 + i * BLK);
            buf[r].v[2 * i + 1] = tree_load<V>(vb1 + i * BLK);
          } else {
            buf[r].v[2 * i] = tree_load<V>(vb0 + i * BLK);
            buf[r].v[2 * i + 1] = tree_load<V>(vb0 + i * BLK + 16 * E);
          }
        }
      };
      auto consume = [&](R& r, int u, float k0, float k1, float v0, float v1) {
        const TreeScale s0 = tree_scale<FP8>(p.scale_log2, k0, v0);
        const TreeScale s1 = PAIR == 2 ? tree_scale<FP8>(p.scale_log2, k1, v1) : s0;
        const int nv = L - (st0 + SP * (u0 + u)) * 32;
        const bool masked = nv < 32;
        uint32_t own = 0xFFFFu;
        if (masked) {  // slots past the sequence hold anything
          own = Tok::registers((1u << nv) - 1u, h);
          tree_keep(r, own);
        }
        tree_step<D, FP8>([&] { return tree_scores(r, qop); }, [] {},
                          [&](int i, int s) { return tree_v(r, i, s); }, s0, s1, masked, own, acc, m_run,
                          l_run);
      };
      // The page ids are waited for here, once.
      asm volatile("" : "+v"(pid0), "+v"(pid1));
      prefetch(0, 0);
      for (int u = 0; u < n; u += 2) {
        prefetch(1, u + 1);
        consume(buf[0], u, ks0[0], ks1[0], vs0[0], vs1[0]);
        // (no way out here: the compiler would wait at the top for what is loaded below)
        prefetch(0, u + 2);
        if (u + 1 < n) consume(buf[1], u + 1, ks0[1], ks1[1], vs0[1], vs1[1]);
      }
    }

    // Drafts (the last stages).  V is turned round through the wave's part of LDS.
    bool odd = false;  // among V of the wave's drafts, something is not finite
    for (int st = a > cache_stages ? a : cache_stages; st < z; ++st) {
      // the wave with the fewest cache steps first
      const int t0 = ((st - cache_stages) * SP + SP - 1 - wave) * 32;
      if (t0 >= nodes) continue;  // uniform in the wave
      uint8_t* vt = (uint8_t*)&s_o[wave][0][0];  // [d][32 nodes]
      odd |= tree_put_drafts<D, 64>(p, vt, b, g, t0, nodes, lane);
      const int t = t0 + ktok < nodes ? t0 + ktok : nodes - 1;  // a row past the nodes is masked
      const uint16_t* kd = p.k_draft + (((int64_t)b * p.num_nodes + t) * Hkv + g) * D;
      auto vf = [&](int i, int s) -> bf16x8 {
        return *(const bf16x8*)(vt + tree_v_at(32 * i + col, Tok::RUN16 ? 2 * h + s : 2 * s + h));
      };
      const TreeScale one{p.scale_log2, 0.f, 1.f, 1.f};
      tree_step<D, FP8>([&] { return tree_draft_scores(kd, p.q + row * D, qop, h); }, [] {}, vf, one, one,
                        true, Tok::registers((uint32_t)(sees >> t0), h), acc, m_run, l_run);
    }

    // The piece's result: the waves' merged in LDS, each summing a share of the quads; then the
    // rows, or one partial.
    const bool whole = a == 0 && z == sq.stages;
    const int64_t slot = 2 * (int64_t)place + (first_piece ? 0 : 1);
    float S = sum_xor32(l_run), M = m_run;
    if (h == 0) s_ml[wave][col] = make_float2(m_run, S);
    if (lane == 0) s_odd[wave] = odd;
    __syncthreads();  // and every wave has done with its drafts
    int any_odd = 0;
#pragma unroll
    for (int w = 0; w < SP; ++w) {
      M = fmaxf(M, s_ml[w][col].x);
      any_odd |= s_odd[w];
    }
    S = 0.f;
#pragma unroll
    for (int w = 0; w < SP; ++w) {
      const float2 ml = s_ml[w][col];
      S += ml.y * (ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M));
    }
    const float f = m_run == M ? 1.f : __builtin_amdgcn_exp2f(m_run - M);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s_o[wave][4 * i + j][lane] = f32x4{acc[i][4 * j] * f, acc[i][4 * j + 1] * f,
                                           acc[i][4 * j + 2] * f, acc[i][4 * j + 3] * f};
    __syncthreads();
    const bool none = L == 0 && sees == 0;  // nothing to attend: zeros
    const float inv = none ? 0.f : 1.f / S;
#pragma unroll
    for (int k = 0; k < QUADS / SP; ++k) {
      const int quad = wave + SP * k, i = quad >> 2, j = quad & 3;
      f32x4 o = s_o[0][quad][lane];
#pragma unroll
      for (int w = 1; w < SP; ++w) o += s_o[w][quad][lane];
      if (!whole)
        ((f32x4*)(p.part_o + slot * 32 * D))[quad * 64 + lane] = o;
      else if (mine)
        *(bf16x4*)(p.out + row * D + 32 * i + 8 * j + 4 * h) =
            bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv),
                   (__bf16)(o[3] * inv)};
    }
    if (__builtin_expect(uni(any_odd), 0)) {
      for (int quad = wave; quad < QUADS; quad += SP) {
        const int d0 = tree_quad_dim(quad, h);
        const f32x4 add = tree_odd_values(p, D, b, g, sees, d0);
        if (!whole)
          tree_add_odd(&((f32x4*)(p.part_o + slot * 32 * D))[quad * 64 + lane], add);
        else if (mine)
          tree_add_odd((bf16x4*)(p.out + row * D + d0), add);
      }
    }
    if (!whole && wave == 0 && h == 0) p.part_ml[slot * 32 + col] = make_float2(M, S);
    if (!whole && a == 0 && tid == 0)
      p.cuts[place] = make_int4(b, g, tree_pieces(rg, place, x + taken + (sq.stages - z) - 1), (int)slot);
    if (p.whole) return;
    x += taken;
    if (x >= rg.x1) return;  // uniform
    first_piece = false;
    while (s_pre[b + 1] <= x) ++b;
    b = uni(b);
    __syncthreads();  // s_o and s_ml: before the next piece's
  }
}

template <int D, int P>
static const void* narrow_fn(bool fp8) {
  return fp8 ? (const void*)&tree_narrow_kernel<D, P, true> : (const void*)&tree_narrow_kernel<D, P, false>;
}

hipError_t launch_tree_narrow(const TreeParams& p, int D, int P, bool fp8, int64_t grid, hipStream_t s) {
  const void* fn = D == 128 ? (P == 16 ? narrow_fn<128, 16>(fp8) : narrow_fn<128, 32>(fp8))
                            : (P == 16 ? narrow_fn<64, 16>(fp8) : narrow_fn<64, 32>(fp8));
  TreeParams arg = p;
  void* args[] = {(void*)&arg};
  const unsigned lds = p.whole ? 0 : (unsigned)(p.num_seqs + 1) * 4;
  return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(64 * kTreeWaves), args, lds, s);
}

}  // namespace dora
