// Which page and which tokens of a sequence a workgroup takes, shared by the kernels
// over the last tokens of each sequence.  Included by HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_internal.h"

namespace dora {

constexpr int kPathMaxPage = 32;  // tokens of a page, at most

// The page that workgroup (b, k) writes: its id (-1: none, or it may not be written,
// then reported), its slots [lo, hi), and for thread i < hi - lo the source row of slot lo + i.
struct PathPage {
  int64_t id;
  int lo, hi, row;
};

__device__ __forceinline__ PathPage path_page(const PathParams& p, int b, int k) {
  PathPage r{-1, 0, 0, 0};
  const int P = p.page_size, L = p.seq_lens[b];
  const int n = p.counts ? p.counts[b] : p.num_tokens;
  if (n == 0) return r;
  bool ok = n > 0 && n <= p.num_tokens && n <= L && (int64_t)L <= (int64_t)p.stride * P;
  if (ok) {
    const int base = L - n, j = base / P + k, t0 = j * P;
    if (t0 >= L) return r;  // no such page
    r.lo = base > t0 ? base - t0 : 0;
    r.hi = L - t0 < P ? L - t0 : P;
    const int i = t0 + r.lo - base + threadIdx.x;  // the token's place in the sequence's list
    r.row = i;  // (loaded beside the page's id, which path_rows waits for)
    if (p.path && (int)threadIdx.x < r.hi - r.lo) r.row = p.path[(int64_t)b * p.num_tokens + i];
    r.id = p.block_table[(int64_t)b * p.stride + j];
    ok = r.id >= 0 && r.id < p.num_pages;
    if (ok && p.page_owner && p.version_ids) ok = p.page_owner[r.id] == p.version_ids[b];
  }
  if (!ok) {
    if (threadIdx.x == 0 && p.dev_status) *p.dev_status = (int32_t)DORA_ERR_DEVICE_CHECK;
    r.id = -1;
  }
  return r;
}

// The source rows of the page's tokens, into s_row; false (for all threads) where one is
// no row: the page is skipped, and reported.
__device__ __forceinline__ bool path_rows(const PathParams& p, const PathPage& pg, int* s_row,
                                          int* s_bad) {
  if (threadIdx.x < 64) {
    const bool mine = (int)threadIdx.x < pg.hi - pg.lo;
    if (mine) s_row[threadIdx.x] = pg.row;
    const bool bad = __any(mine && (pg.row < 0 || pg.row >= p.num_tokens));
    if (threadIdx.x == 0) *s_bad = bad;
  }
  __syncthreads();
  if (!*s_bad) return true;
  if (threadIdx.x == 0 && p.dev_status) *p.dev_status = (int32_t)DORA_ERR_DEVICE_CHECK;
  return false;
}

// Launches over (page, sequence): f(parameters, grid, first sequence) for the sequences of a grid at a time.  The pages of a
// sequence are neighbours, so that a long run's go to all XCDs (workgroups go to them in turn).
template <typename F>
inline hipError_t each_launch(const PathParams& p, F f) {
  constexpr int SEQS = 32768;
  // pages that p.num_tokens tokens can touch
  const unsigned pages = (unsigned)((p.num_tokens + p.page_size - 2) / p.page_size + 1);
  const int64_t row = (int64_t)p.num_tokens * p.num_kv_heads * p.head_dim;
  for (int first = 0; first < p.num_seqs; first += SEQS) {
    PathParams q = p;
    q.num_seqs = p.num_seqs - first < SEQS ? p.num_seqs - first : SEQS;
    if (p.k_new) q.k_new += first * row;
    if (p.v_new) q.v_new += first * row;
    if (p.path) q.path += (int64_t)first * p.num_tokens;
    if (p.counts) q.counts += first;
    q.block_table += (int64_t)first * p.stride;
    q.seq_lens += first;
    if (p.version_ids) q.version_ids += first;
    const hipError_t e = f(q, dim3(pages, (unsigned)q.num_seqs), first);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace dora
