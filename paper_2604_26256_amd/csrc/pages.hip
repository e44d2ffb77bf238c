// Decode attention over a list of pages for each (sequence, KV head): what a selection
// names, or, of 4-bit pages without lists, all pages of a short row.
//
// Bound by memory: each listed page is read once, by one wave, straight into matrix operands
// (16 query columns: a KV head's group), two steps of loads in flight.  In a stream of calls, where one's start
// covers the other's end, 512 lists of 2,048 tokens in bf16 (537 MB) take 86 us, 6.2 TB/s (89 to 93 in
// a trace, which runs kernels one by one); 4,000 fp8 lists of up to 3,200 tokens (2.65 GB) 433 us, 6.1; 1,024
// 4-bit lists of 2,560 tokens of 128 dims in pages of 16 (347 MB) 70 us, 4.9 (72 to 75), where pages of 32
// take 59, 5.8: a tile of 16 such tokens is 1,088 bytes, half a line more than whole ones, and the rate
// of tiles read here and there falls with their size.  Reading lists beside lengths and counts, one wait
// fewer at the start, changed nothing: what runs beside a start hides it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bits_core.h"
#include "decode_core.h"
#include "fp4_core.h"
#include "merge_core.h"
#include "pages_internal.h"
#include "tree_core.h"

namespace dora {

// The listed pages of a workgroup's chunk, in LDS: page ids and how many of a page's tokens count.
// An entry that is no page of the sequence has none, and id 0 (its table entry is not read).
struct PagesStage {
  int id[kPagesMaxChunk];
  int tokens[kPagesMaxChunk];
};

// Entries of segment (b, g)'s list.
__device__ __forceinline__ int pages_listed(const PagesParams& p, int seg, int L) {
  if (!p.lists) return pages_of(L, p.page_size, p.stride);
  const int n = p.counts[seg];
  return n < 0 ? 0 : n < p.list_stride ? n : p.list_stride;
}

template <int P>
__device__ __forceinline__ void pages_stage(const PagesParams& p, PagesStage& s, int seg, int b, int L,
                                            int first, int n) {
  const int32_t* row = p.block_table + (int64_t)b * p.stride;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int j = p.lists ? p.lists[(int64_t)seg * p.list_stride + first + i] : first + i;
    int tokens = 0, id = 0;
    if (j >= 0 && j < p.stride && (int64_t)j * P < L) {
      tokens = L - j * P < P ? L - j * P : P;
      id = row[j];
    }
    s.id[i] = id;
    s.tokens[i] = tokens;
  }
  __syncthreads();
}

// What a wave holds of a segment after its pages, into LDS; then the workgroup's merge of its
// waves, and the output rows or, where the segment has further chunks, a partial.
template <int D, int WAVES>
struct PagesMerge {
  float o[WAVES][16][D + 4];
  float2 ml[WAVES][16];
  int any[WAVES];  // whether a token counted
};

template <int D, int WAVES>
__device__ __forceinline__ void pages_finish(const PagesParams& p, PagesMerge<D, WAVES>& s,
                                             const f32x4 (&acc)[D / 16], float m_run, float l_run,
                                             bool any, int seg, int64_t row0, int c, bool cut) {
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4, G = p.group;
  const float l_tot = sum_xor32(sum_xor16(l_run));
  if (col < G) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *(f32x4*)&s.o[wave][col][16 * i + 4 * grp] = acc[i];
    if (grp == 0) s.ml[wave][col] = make_float2(m_run, l_tot);
  }
  if (lane == 0) s.any[wave] = any;
  __syncthreads();
  bool some = false;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) some = some || s.any[w];
  for (int e = threadIdx.x; e < G * (D / 4); e += 64 * WAVES) {
    const int h = e / (D / 4), d4 = e - h * (D / 4);
    float M = kNoMax, S = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      if (s.any[w]) M = fmaxf(M, s.ml[w][h].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (!s.any[w]) continue;
      const float2 ml = s.ml[w][h];
      const float f = ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
      S += f * ml.y;
      o += f * *(const f32x4*)&s.o[w][h][4 * d4];
    }
    if (cut) {  // uniform: one of several chunks
      const int64_t slot = ((int64_t)seg * p.chunks + c) * G + h;
      *(f32x4*)(p.part_o + slot * D + 4 * d4) = o;
      if (d4 == 0) p.part_ml[slot] = make_float2(some ? M : -__builtin_inff(), S);
    } else {
      const float inv = some ? 1.f / S : 0.f;  // a row that attends nothing is 0
      *(bf16x4*)(p.out + (row0 + h) * D + 4 * d4) =
          bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv),
                 (__bf16)(o[3] * inv)};
    }
  }
}

// One workgroup of WAVES waves per (sequence, KV head) segment, or per chunk of
// p.chunk_pages of its listed pages.  bf16 and fp8 pages; a step is one page.
template <int D, int P, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void pages_kernel(PagesParams p) {
  constexpr int DBLK = D / 16, TILE_BYTES = P * D * (FP8 ? 1 : 2);
  __shared__ __align__(16) union {
    PagesStage stage;
    PagesMerge<D, WAVES> merge;
  } s;
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int Hkv = p.num_kv_heads, G = p.group;
  const int c = (int)blockIdx.y, seg = (int)blockIdx.x;
  const int b = seg / Hkv, g = seg - b * Hkv;
  const int64_t row0 = (int64_t)b * p.num_q_heads + (int64_t)g * G;
  const int64_t most = (int64_t)p.stride * P;
  int L = uni(p.seq_lens[b]);
  L = L < most ? L : (int)most;  // a contract violation stays in bounds
  const int n_seg = uni(pages_listed(p, seg, L)), u0 = c * p.chunk_pages;
  if (c > 0 && u0 >= n_seg) return;  // uniform
  const int n = n_seg - u0 < p.chunk_pages ? n_seg - u0 : p.chunk_pages;
  bf16x8 qop[D / 32];
  load_q_operand<D, FP8>(qop, p.q + (row0 + col) * D, col < G);
  pages_stage<P>(p, s.stage, seg, b, L, u0, n);

  f32x4 acc[DBLK];
#pragma unroll
  for (int i = 0; i < DBLK; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;
  bool any = false;
  const int steps = (n - wave + WAVES - 1) / WAVES;  // <= 0: none for this wave
  if (steps > 0) {
    const uint32_t koff = step_koff<D, P, P>(col, grp), voff = step_voff<D, P, FP8, P>(col, grp);
    PageRegs<D, P, FP8> buf[2];
    float s_ks[2] = {1.f, 1.f}, s_vs[2] = {1.f, 1.f};
    int tokens[2];
    auto prefetch = [&](int r, int u) {
      const bool past = u >= steps;  // past the last step the loads still issue, one line each
      const int i = wave + WAVES * (past ? steps - 1 : u);
      const int page = uni(s.stage.id[i]);
      tokens[r] = uni(s.stage.tokens[i]);
      if constexpr (FP8) {
        s_ks[r] = p.k_scales[page];
        s_vs[r] = p.v_scales[page];
      }
      const int64_t at = (int64_t)page * p.page_bytes + (int64_t)g * TILE_BYTES;
      load_step<D, P, FP8, P, true>(buf[r], p.k_pages, p.v_pages, at, at, past ? 0u : koff,
                                    past ? 0u : voff);
    };
    prefetch(0, 0);
    int u = 0;
    while (true) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        prefetch(r ^ 1, u + 1);
        if (tokens[r] > 0) {  // uniform
          any = true;
          const uint32_t bits = tokens[r] >= 32 ? ~0u : (1u << tokens[r]) - 1u;
          consume_bits<D, P, FP8>(buf[r], bits, tree_scale<FP8>(p.scale_log2, s_ks[r], s_vs[r]), qop,
                                  acc, m_run, l_run);
        }
        if (++u >= steps) goto done;
      }
    }
  }
done:
  __syncthreads();  // the stage is done with
  pages_finish<D>(p, s.merge, acc, m_run, l_run, any, seg, row0, c, n_seg > p.chunk_pages);
}

// The same over 4-bit pages; a step is 64 tokens.
template <int D, int P, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 3) void pages4_kernel(PagesParams p) {
  typedef Fp4<D, P> F;
  constexpr int DBLK = D / 16;
  __shared__ __align__(16) union {
    PagesStage stage;
    PagesMerge<D, WAVES> merge;
  } s;
  __shared__ bf16x8 s_q[D / 32][64];
  const int lane = threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6);
  const int col = lane & 15;
  const int Hkv = p.num_kv_heads, G = p.group;
  const int c = (int)blockIdx.y, seg = (int)blockIdx.x;
  const int b = seg / Hkv, g = seg - b * Hkv;
  const int64_t row0 = (int64_t)b * p.num_q_heads + (int64_t)g * G;
  const int64_t most = (int64_t)p.stride * P;
  int L = uni(p.seq_lens[b]);
  L = L < most ? L : (int)most;
  const int n_seg = uni(pages_listed(p, seg, L)), u0 = c * p.chunk_pages;
  if (c > 0 && u0 >= n_seg) return;  // uniform
  const int n = n_seg - u0 < p.chunk_pages ? n_seg - u0 : p.chunk_pages;
  if (wave == 0) {  // (in registers the rows would cost the third workgroup of a CU)
    typename F::Query q;
    F::load_query(q, p.q + (row0 + col) * D, col < G);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s_q[i][lane] = q[i];
  }
  pages_stage<P>(p, s.stage, seg, b, L, u0, n);

  f32x4 acc[DBLK];
#pragma unroll
  for (int i = 0; i < DBLK; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoMax, l_run = 0.f;
  bool any = false;
  const int n_steps = (n + F::PAGES - 1) / F::PAGES;
  const int steps = (n_steps - wave + WAVES - 1) / WAVES;
  if (steps > 0) {
    const uint32_t koff = F::k_off(lane), ksoff = F::k_scale_off(lane), voff = F::v_off(lane),
                   vsoff = F::v_scale_off(lane);
    const int64_t tile = (int64_t)g * F::TILE;
    typename F::Regs buf[2];
    int nv[2];
    auto prefetch = [&](int r, int u) {
      // (past the last step it is loaded again: under a branch the loads would be waited for together)
      const int i = F::PAGES * (wave + WAVES * (u < steps ? u : steps - 1)), last = n - 1;
      const int ik = i + F::k_page(lane), iv = i + F::v_page(lane);  // past the end: no tokens
      const int64_t k = s.stage.id[ik < n ? ik : last], v = s.stage.id[iv < n ? iv : last];
      nv[r] = iv < n ? s.stage.tokens[iv] - F::group_slot(lane) : 0;
      F::load(buf[r], p.k_pages + k * p.page_bytes + tile, p.v_pages + v * p.page_bytes + tile, koff,
              ksoff, voff, vsoff);
    };
    prefetch(0, 0);
    int u = 0;
    while (true) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        prefetch(r ^ 1, u + 1);
        const bool all = !__ballot(nv[r] < 16);
        if (all || __ballot(nv[r] > 0)) {
          any = true;
          F::consume(buf[r], all, nv[r], p.scale_log2, [&](int i) { return s_q[i][lane]; }, acc, m_run,
                     l_run);
        }
        if (++u >= steps) goto done;
      }
    }
  }
done:
  __syncthreads();
  pages_finish<D>(p, s.merge, acc, m_run, l_run, any, seg, row0, c, n_seg > p.chunk_pages);
}

// Merges the chunks of a segment that has more than one, for the tasks part * per .. of it.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_combine_kernel(PagesParams p, int per) {
  const int seg = (int)blockIdx.x;
  const int b = seg / p.num_kv_heads, g = seg - b * p.num_kv_heads;
  const int64_t most = (int64_t)p.stride * p.page_size;
  const int len = p.seq_lens[b], L = len < most ? len : (int)most;
  const int n = pages_listed(p, seg, L);
  if (n <= p.chunk_pages) return;
  const int64_t slot0 = (int64_t)seg * p.chunks;
  merge_segment<THREADS, true>(p.part_o, p.part_ml, p.out, p.num_q_heads, p.group, p.head_dim, b, g,
                               (int)blockIdx.y * per, per, (n + p.chunk_pages - 1) / p.chunk_pages,
                               [=](int k) { return slot0 + k; });
}

// DORA_FLAG_VALIDATE: lengths, counts, entries, and the ids and owners of the listed pages.
__global__ __launch_bounds__(256) void pages_validate_kernel(ValidateParams p, const int32_t* lists,
                                                             const int32_t* counts, int num_kv_heads,
                                                             int list_stride) {
  const int seg = blockIdx.x, b = seg / num_kv_heads;
  const int L = p.seq_lens[b], n = counts[seg];
  if (L < 0 || (int64_t)L > (int64_t)p.stride * p.page_size || n < 0 || n > list_stride) {
    if (threadIdx.x == 0) atomicOr(p.err, 1);
    return;
  }
  const int pages = (int)(((int64_t)L + p.page_size - 1) / p.page_size);
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int j = lists[(int64_t)seg * list_stride + i];
    if (j < 0 || j >= pages) {
      atomicOr(p.err, 8);
      continue;
    }
    const int32_t id = p.block_table[(int64_t)b * p.stride + j];
    if (id < 0 || id >= p.num_pages)
      atomicOr(p.err, 2);
    else if (p.page_owner && p.page_owner[id] != p.version_ids[b])
      atomicOr(p.err, 4);
  }
}

template <int D, int P, int WAVES>
static const void* pages_fn(int kv_dtype) {
  return kv_dtype == DORA_KV_FP4        ? (const void*)&pages4_kernel<D, P, WAVES>
         : kv_dtype == DORA_KV_FP8_E4M3 ? (const void*)&pages_kernel<D, P, true, WAVES>
                                        : (const void*)&pages_kernel<D, P, false, WAVES>;
}
template <int WAVES>
static const void* pages_fn(int kv_dtype, int head_dim, int page_size) {
  return head_dim == 128
             ? (page_size == 16 ? pages_fn<128, 16, WAVES>(kv_dtype) : pages_fn<128, 32, WAVES>(kv_dtype))
             : (page_size == 16 ? pages_fn<64, 16, WAVES>(kv_dtype) : pages_fn<64, 32, WAVES>(kv_dtype));
}

hipError_t launch_pages(const PagesParams& p, int kv_dtype, hipStream_t s) {
  const void* fn = p.waves == 1 ? pages_fn<1>(kv_dtype, p.head_dim, p.page_size)
                                : pages_fn<kSegWaves>(kv_dtype, p.head_dim, p.page_size);
  PagesParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(fn, dim3((unsigned)(p.num_seqs * p.num_kv_heads), (unsigned)p.chunks),
                         dim3(64u * (unsigned)p.waves), args, 0, s);
}

hipError_t launch_pages_combine(const PagesParams& p, hipStream_t s) {
  const int segs = p.num_seqs * p.num_kv_heads;
  const int tasks = p.group * (p.head_dim / 4);
  int parts = 1;  // as launch_combine_chunks
  while (tasks > 64 * parts && p.chunks * (tasks / parts) > 8 * 512 && 2 * parts * segs <= 1024)
    parts *= 2;
  hipLaunchKernelGGL(pages_combine_kernel<512>, dim3((unsigned)segs, (unsigned)parts), dim3(512), 0, s,
                     p, (tasks + parts - 1) / parts);
  return hipGetLastError();
}

hipError_t launch_pages_validate(const ValidateParams& p, const int32_t* lists, const int32_t* counts,
                                 int num_kv_heads, int list_stride, hipStream_t s) {
  hipLaunchKernelGGL(pages_validate_kernel, dim3((unsigned)(p.num_seqs * num_kv_heads)), dim3(256), 0,
                     s, p, lists, counts, num_kv_heads, list_stride);
  return hipGetLastError();
}

}  // namespace dora
