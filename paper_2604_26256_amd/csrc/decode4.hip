// Decode attention over 4-bit pages: stream-K over the batch's (sequence, KV head, step of 64
// tokens) work, as decode.hip has it over page-heads.  Every wavefront takes an equal
// contiguous range; the pieces of the segments that the ranges cut are joined by decode.hip's
// combine.
//
// Bound by memory, 17 / 32 byte a value: 256 rows of 8 KV heads (1.67 GB) 286 us with the combine, 5.9
// TB/s; 64 rows of 4 KV heads (126 MB) 38.7 us, of which 6 are the combine and about 10 the
// start: lengths, ids, first pages, one after another.  One wave a SIMD has 512 registers for two
// steps of pages (17 KB) and its sums; a third step in flight was no faster (the loads of 1,024 waves, 18 MB,
// already cover the latency), nor were more waves (api.cpp, decode_waves).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode_core.h"
#include "dora_internal.h"
#include "fp4_core.h"
#include "ranges_core.h"

namespace dora {

// Steps of a sequence whose table holds at most stride * P tokens.
__device__ __forceinline__ int steps4_of(int L, int P, int stride) {
  const int64_t most = (int64_t)stride * P;
  const int n = L < 0 ? 0 : L < most ? L : (int)most;  // a contract violation stays in bounds
  return (int)(((int64_t)n + kFp4Step - 1) / kFp4Step);
}

template <int D, int P, int NBUF>
__global__ __launch_bounds__(64, 2) void decode4_kernel(DecodeParams p) {
  typedef Fp4<D, P> F;
  constexpr int DBLK = D / 16;
  extern __shared__ int sN[];  // steps of a KV head before each sequence, [B + 1]
  const int lane = threadIdx.x, col = lane & 15, grp = lane >> 4;
  const int B = p.num_seqs, Hkv = p.num_kv_heads, G = p.group, Hq = p.num_q_heads;

  int carry = 0;
  for (int base = 0; base < B; base += 64 * 8) {
    int n[8], tsum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // (no branch around the loads, so that they issue together)
      const int b = base + lane * 8 + k;
      const int L = p.seq_lens[b < B ? b : B - 1];
      n[k] = b < B ? steps4_of(L, P, p.stride) : 0;
      tsum += n[k];
    }
    const int incl = wave_inclusive_scan(tsum);
    int excl = carry + incl - tsum;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int b = base + lane * 8 + k;
      if (b < B) sN[b] = excl;
      excl += n[k];
    }
    carry += __shfl(incl, 63);
  }
  if (lane == 0) sN[B] = carry;
  __syncthreads();
  const int64_t w = blockIdx.x;
  for (int b = (int)w; b < B; b += gridDim.x) {  // empty sequences, shared out
    if (sN[b + 1] != sN[b]) continue;
    uint32_t* o = (uint32_t*)(p.out + (int64_t)b * Hq * D);
    for (int e = lane; e < Hq * D / 2; e += 64) o[e] = 0u;
    if (p.seg_records)
      for (int e = lane; e < Hkv; e += 64) p.cuts[(int64_t)b * Hkv + e] = make_int4(-1, 0, 0, 0);
  }

  const int T = uni(Hkv * carry);  // fits 32 bits: the host bounds batch x stride x Hkv
  const int W = uni(effective_waves(T, (int)gridDim.x, p.min_range));
  if (T == 0 || w >= W) {
    if (lane == 0 && !p.seg_records) p.cuts[w] = make_int4(-1, 0, 0, 0);
    return;
  }
  Split split;
  split.q = uni(T / W);
  split.rem = T - split.q * W;
  const int x0 = split.begin((int)w), x1 = split.begin((int)w + 1);

  // A place in the work list: sequence, KV head, step, steps of the sequence.
  struct Place {
    int b, g, u, n, L;
  };
  // (by scalar loads: a vector load would be waited for together with the pages under way)
  typedef __attribute__((address_space(4))) const int32_t constant_i32;
  constant_i32* lens = (constant_i32*)(uintptr_t)p.seq_lens;
  auto at_sequence = [&](Place& c) {
    c.n = uni(sN[c.b + 1] - sN[c.b]);
    c.L = lens[c.b];
    const int64_t most = (int64_t)p.stride * P;
    if (c.L > most) c.L = (int)most;
  };
  auto next = [&](Place& c) {
    if (++c.u < c.n) return;
    c.u = 0;
    if (++c.g < Hkv) return;
    c.g = 0;
    do ++c.b; while (c.b < B && uni(sN[c.b + 1] - sN[c.b]) == 0);
    if (c.b < B) at_sequence(c);
  };
  Place ids, page, here;  // of the next ids, the next pages, the step that is consumed
  {
    int lo = 0, hi = B;  // the last b with Hkv * N(b) <= x0
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (Hkv * sN[mid] <= x0) lo = mid; else hi = mid;
    }
    here.b = uni(lo);
    at_sequence(here);
    const int r = x0 - Hkv * sN[here.b];
    here.g = uni(r / here.n);
    here.u = uni(r - here.g * here.n);
    page = ids = here;
  }

  const uint32_t koff = F::k_off(lane), ksoff = F::k_scale_off(lane), voff = F::v_off(lane),
                 vsoff = F::v_scale_off(lane);
  int kid, vid;  // page ids of the lane's tiles
  auto load_ids = [&](const Place& c, int& k, int& v) {
    const int last = (c.L + P - 1) / P - 1, j = c.u * F::PAGES;  // past the end: the last page again
    const int jk = j + F::k_page(lane), jv = j + F::v_page(lane);
    const int32_t* row = p.block_table + (int64_t)c.b * p.stride;
    k = row[jk < last ? jk : last];
    v = row[jv < last ? jv : last];
  };
  auto load_pages = [&](const Place& c, typename F::Regs& r, int k, int v) {
    const int64_t tile = (int64_t)c.g * F::TILE;
    F::load(r, p.k_pages + (int64_t)k * p.page_bytes + tile,
            p.v_pages + (int64_t)v * p.page_bytes + tile, koff, ksoff, voff, vsoff);
  };

  f32x4 acc[DBLK];
  typename F::Query q;
  float m_run = kNoMax, l_run = 0.f;
  bool whole = false, begun_here = false, first_seg = true;
  int4 cut = make_int4(-1, 0, 0, 0);

  auto finish = [&]() {
    const float l_tot = sum_xor32(sum_xor16(l_run));
    if (col < G) {
      if (whole) {
        const float inv = 1.f / l_tot;
        uint16_t* o = p.out + ((int64_t)here.b * Hq + here.g * G + col) * D + 4 * grp;
#pragma unroll
        for (int i = 0; i < DBLK; ++i)
          *(bf16x4*)(o + 16 * i) = bf16x4{(__bf16)(acc[i][0] * inv), (__bf16)(acc[i][1] * inv),
                                          (__bf16)(acc[i][2] * inv), (__bf16)(acc[i][3] * inv)};
      } else {
        const int64_t slot = 2 * w + (first_seg ? 0 : 1);
        float* po = p.part_o + (slot * G + col) * D + 4 * grp;
#pragma unroll
        for (int i = 0; i < DBLK; ++i) *(f32x4*)(po + 16 * i) = acc[i];
        if (grp == 0) p.part_ml[slot * G + col] = make_float2(m_run, l_tot);
      }
    }
    if (!whole && begun_here) {  // pieces: ranges w .. the range of the segment's last step
      const int s0 = Hkv * sN[here.b] + here.g * here.n;
      cut = make_int4(here.b, here.g, split.range_of(s0 + here.n - 1) - (int)w + 1, first_seg ? 0 : 1);
    }
    if (p.seg_records && lane == 0 && (whole || begun_here))
      p.cuts[(int64_t)here.b * Hkv + here.g] =
          whole ? make_int4(-1, 0, 0, 0) : make_int4((int)w, cut.z, cut.w, 0);
    first_seg = false;
  };

  // The ids of a step are loaded one step before its pages, the pages NBUF - 1 steps before they are used.  Behind the
  // range's end the loads are made again: under a branch they would be waited for with those before them; for the
  // same reason the loads before the loop come in the loop's order.
  typename F::Regs buf[NBUF];
  int left_ids = x1 - x0 - 1, left_pages = x1 - x0 - 1;  // steps that are behind `ids` and `page`
  auto advance = [&](Place& c, int& left) {
    if (left > 0) {
      --left;
      next(c);
    }
  };
  load_ids(ids, kid, vid);
#pragma unroll
  for (int i = 0; i < NBUF - 1; ++i) {
    const int k = kid, v = vid;
    if (i > 0) advance(page, left_pages);
    advance(ids, left_ids);
    load_ids(ids, kid, vid);
    load_pages(page, buf[i], k, v);
  }
  int x = x0;
  while (true) {
#pragma unroll
    for (int r = 0; r < NBUF; ++r) {
      if (x == x0 || here.u == 0) {
        whole = begun_here = here.u == 0;
        m_run = kNoMax;
        l_run = 0.f;
#pragma unroll
        for (int i = 0; i < DBLK; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        F::load_query(q, p.q + ((int64_t)here.b * Hq + (int64_t)here.g * G + col) * D, col < G);
        // waited for here, before the next pages' loads: after the branch it would be with them
#pragma unroll
        for (int i = 0; i < D / 32; ++i) asm volatile("" : "+v"(q[i]));
      }
      const int k = kid, v = vid;
      advance(page, left_pages);
      advance(ids, left_ids);
      load_ids(ids, kid, vid);
      load_pages(page, buf[(r + NBUF - 1) % NBUF], k, v);
      const int left = here.L - here.u * kFp4Step;
      F::consume(buf[r], left >= kFp4Step, left - 16 * grp, p.scale_log2, [&](int s) { return q[s]; }, acc,
                 m_run, l_run);
      const bool last = here.u == here.n - 1;
      if (last || x == x1 - 1) {
        whole = whole && last;
        finish();
      }
      if (++x >= x1) goto done;
      next(here);
    }
  }
done:
  if (lane == 0 && !p.seg_records) p.cuts[w] = cut;
}

static const void* decode4_symbol(int head_dim, int page_size) {
  if (head_dim == 128)
    return page_size == 16 ? (const void*)&decode4_kernel<128, 16, 2> : (const void*)&decode4_kernel<128, 32, 2>;
  return page_size == 16 ? (const void*)&decode4_kernel<64, 16, 2> : (const void*)&decode4_kernel<64, 32, 2>;
}

hipError_t launch_decode4(const DecodeParams& p, int head_dim, int page_size, int64_t waves,
                          hipStream_t s) {
  if (waves <= 0) return hipSuccess;
  DecodeParams arg = p;
  void* args[] = {(void*)&arg};
  return hipLaunchKernel(decode4_symbol(head_dim, page_size), dim3((unsigned)waves), dim3(64), args,
                         decode_lds_bytes(p.num_seqs), s);
}

}  // namespace dora
