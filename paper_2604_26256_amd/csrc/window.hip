// Decode attention with a sliding window and sinks: token t of a sequence of L counts
// where t < sinks or t >= L - window.  Only the pages that hold such tokens are read;
// the table's other entries are not looked at, so their pages may be free.
//
// Bound by memory: each visible page is read once, by one wave, straight into the
// operands of 16x16 matrix products (16 query columns: a KV head's group), two steps of
// loads in flight.  512 rows of up to 65,536 tokens in bf16 through a window of 1,024 and 4
// sinks (64 query heads, 8 KV heads of 128 dims): 1.6 GB in 276 us, 5.8 TB/s.  500 rows in
// fp8 through 4,090 and 20: 3.2 GB in 536 us, 5.9 TB/s (a large copy: 6.6).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"
#include "decode_core.h"
#include "merge_core.h"
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

// Bits of page j's P tokens that count.
template <int P>
__device__ __forceinline__ uint32_t page_bits(int j, int L, int begin, int sinks) {
  const int t0 = j * P;
  auto upto = [](int k) { return k <= 0 ? 0u : k >= 32 ? ~0u : (1u << k) - 1u; };
  constexpr uint32_t ALL = P == 32 ? ~0u : 0xFFFFu;
  return (~upto(begin - t0) | upto(sinks - t0)) & upto(L - t0) & ALL;
}

// One workgroup of kSegWaves waves per (sequence, KV head) segment, or per chunk of
// p.chunk_pages of its visible pages.  Wave w takes pages w, w + kSegWaves, ...; lane u holds the
// id of the wave's u-th page.  (Two 16-token pages a step, as the plain decode has for few
// segments, gain 3% for 16 segments of 512 tokens, 64 dims, nothing for 512, and lose 6% for 1,024.)
template <int D, int P, bool FP8>
__global__ __launch_bounds__(64 * kSegWaves, 2) void window_kernel(WindowParams p) {
  constexpr int KSTEPS = D / 32, DBLK = D / 16;
  constexpr int TILE_BYTES = P * D * (FP8 ? 1 : 2);
  constexpr int ROW = D + 4;
  __shared__ __align__(16) float s_o[kSegWaves][16][ROW];
  __shared__ float2 s_ml[kSegWaves][16];

  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int Hkv = p.num_kv_heads, G = p.group;
  const int c = (int)blockIdx.y, seg = (int)blockIdx.x;
  const int b = seg / Hkv, g = seg - b * Hkv;
  const int64_t row0 = (int64_t)b * p.num_q_heads + (int64_t)g * G;
  const int L = uni(p.seq_lens[b]);
  bf16x8 qop[KSTEPS];
  load_q_operand<D, FP8>(qop, p.q + (row0 + col) * D, col < G);

  const Visible vis = visible_pages(L, P, p.stride, p.window, p.sinks);
  const int n_seg = vis.pages(), u0 = c * p.chunk_pages;
  if (c > 0 && u0 >= n_seg) return;  // uniform: the segment ends before this chunk
  const int n = n_seg - u0 < p.chunk_pages ? n_seg - u0 : p.chunk_pages;
  const int Lc = (int64_t)L < (int64_t)p.stride * P ? L : p.stride * P;
  const int begin = Lc > p.window ? Lc - p.window : 0;
  auto page_at = [&](int u) { return u < vis.sink ? u : vis.first + (u - vis.sink); };
  f32x4 acc[DBLK];
#pragma unroll
  for (int i = 0; i < DBLK; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;
  const int steps = (n - wave + kSegWaves - 1) / kSegWaves;  // <= 0: none for this wave
  if (steps > 0) {
    // this lane's page of the wave (the last one past the end)
    const int ul = wave + kSegWaves * lane;
    const int j = page_at(u0 + (ul < n ? ul : n - 1));
    int pid = p.block_table[(int64_t)b * p.stride + j];
    const int bits = (int)page_bits<P>(j, Lc, begin, p.sinks);
    const uint32_t koff = step_koff<D, P, P>(col, grp), voff = step_voff<D, P, FP8, P>(col, grp);
    PageRegs<D, P, FP8> buf[2];
    float s_ks[2] = {1.f, 1.f}, s_vs[2] = {1.f, 1.f};
    auto prefetch = [&](int r, int u) {
      const bool past = u >= steps;  // past the last step the loads still issue, one line each
      u = past ? steps - 1 : u;
      const int page = __builtin_amdgcn_readlane(pid, u);
      if constexpr (FP8) {
        s_ks[r] = p.k_scales[page];
        s_vs[r] = p.v_scales[page];
      }
      const int64_t at = (int64_t)page * p.page_bytes + (int64_t)g * TILE_BYTES;
      load_step<D, P, FP8, P, true>(buf[r], p.k_pages, p.v_pages, at, at, past ? 0u : koff,
                                    past ? 0u : voff);
    };
    // The table entries are waited for here, once.
    asm volatile("" : "+v"(pid));
    prefetch(0, 0);
    int u = 0;
    while (true) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        prefetch(r ^ 1, u + 1);
        const uint32_t m = (uint32_t)__builtin_amdgcn_readlane(bits, u);
        consume_bits<D, P, FP8>(buf[r], m, tree_scale<FP8>(p.scale_log2, s_ks[r], s_vs[r]), qop, acc,
                                m_run, l_run);
        if (++u >= steps) goto done;
      }
    }
  }
done:
  const float l_tot = sum_xor32(sum_xor16(l_run));
  if (col < G) {
#pragma unroll
    for (int i = 0; i < DBLK; ++i) *(f32x4*)&s_o[wave][col][16 * i + 4 * grp] = acc[i];
    if (grp == 0) s_ml[wave][col] = make_float2(m_run, l_tot);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * (D / 4); e += 64 * kSegWaves) {
    const int h = e / (D / 4), d4 = e - h * (D / 4);
    float M = s_ml[0][h].x, S = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 1; w < kSegWaves; ++w) M = fmaxf(M, s_ml[w][h].x);
#pragma unroll
    for (int w = 0; w < kSegWaves; ++w) {
      if (w >= n) break;  // uniform: waves past the pages hold nothing
      const float2 ml = s_ml[w][h];
      const float f = ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
      S += f * ml.y;
      o += f * *(const f32x4*)&s_o[w][h][4 * d4];
    }
    if (n_seg > p.chunk_pages) {  // uniform: one of several chunks
      const int64_t slot = ((int64_t)seg * p.chunks + c) * G + h;
      *(f32x4*)(p.part_o + slot * D + 4 * d4) = o;
      if (d4 == 0) p.part_ml[slot] = make_float2(M, S);
    } else {
      const float inv = n > 0 ? 1.f / S : 0.f;  // an empty sequence gives zeros
      *(bf16x4*)(p.out + (row0 + h) * D + 4 * d4) =
          bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv),
                 (__bf16)(o[3] * inv)};
    }
  }
}

// Merges the chunks of a segment that has more than one.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void window_combine_kernel(WindowParams p, int per) {
  const int seg = (int)blockIdx.x;
  const int b = seg / p.num_kv_heads, g = seg - b * p.num_kv_heads;
  const int n = visible_pages(p.seq_lens[b], p.page_size, p.stride, p.window, p.sinks).pages();
  if (n <= p.chunk_pages) return;
  const int64_t slot0 = (int64_t)seg * p.chunks;
  merge_segment<THREADS>(p.part_o, p.part_ml, p.out, p.num_q_heads, p.group, p.head_dim, b, g,
                         (int)blockIdx.y * per, per, (n + p.chunk_pages - 1) / p.chunk_pages,
                         [=](int k) { return slot0 + k; });
}

// DORA_FLAG_VALIDATE: the lengths, and the ids and owners of the visible pages.
__global__ __launch_bounds__(256) void window_validate_kernel(ValidateParams p, int window, int sinks) {
  const int b = blockIdx.x;
  const int L = p.seq_lens[b];
  if (L < 0 || (int64_t)L > (int64_t)p.stride * p.page_size) {
    if (threadIdx.x == 0) atomicOr(p.err, 1);
    return;
  }
  const Visible vis = visible_pages(L, p.page_size, p.stride, window, sinks);
  const int32_t* bt = p.block_table + (int64_t)b * p.stride;
  for (int u = threadIdx.x; u < vis.pages(); u += blockDim.x) {
    const int32_t pid = bt[u < vis.sink ? u : vis.first + (u - vis.sink)];
    if (pid < 0 || pid >= p.num_pages)
      atomicOr(p.err, 2);
    else if (p.page_owner && p.page_owner[pid] != p.version_ids[b])
      atomicOr(p.err, 4);
  }
}

template <int D, int P>
static const void* window_fn(bool fp8) {
  return fp8 ? (const void*)&window_kernel<D, P, true> : (const void*)&window_kernel<D, P, false>;
}

hipError_t launch_window(const WindowParams& p, bool fp8, hipStream_t s) {
  const void* fn = p.head_dim == 128
                       ? (p.page_size == 16 ? window_fn<128, 16>(fp8) : window_fn<128, 32>(fp8))
                       : (p.page_size == 16 ? window_fn<64, 16>(fp8) : window_fn<64, 32>(fp8));
  WindowParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)(p.num_seqs * p.num_kv_heads), (unsigned)p.chunks),
                         dim3(64 * kSegWaves), args, 0, s);
}

hipError_t launch_window_combine(const WindowParams& p, hipStream_t s) {
  const int segs = p.num_seqs * p.num_kv_heads;
  const int tasks = p.group * (p.head_dim / 4);
  int parts = 1;  // as launch_combine_chunks
  while (tasks > 64 * parts && p.chunks * (tasks / parts) > 8 * 512 && 2 * parts * segs <= 1024)
    parts *= 2;
  hipLaunchKernelGGL(window_combine_kernel<512>, dim3((unsigned)segs, (unsigned)parts), dim3(512), 0,
                     s, p, (tasks + parts - 1) / parts);
  return hipGetLastError();
}

hipError_t launch_window_validate(const ValidateParams& p, int window, int sinks, hipStream_t s) {
  hipLaunchKernelGGL(window_validate_kernel, dim3(p.num_seqs), dim3(256), 0, s, p, window, sinks);
  return hipGetLastError();
}

}  // namespace dora
