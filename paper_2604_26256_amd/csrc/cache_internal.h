// Internal declarations of the operators around the cache (tree and window
// attention, path append, page copies).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dora.h"
#include "dora_internal.h"

namespace dora {

// Tree attention.
constexpr int kTreeWaves = 4;        // waves of a workgroup (with two tiles: two)
constexpr int kTreeMaxSeqs = 2048;   // sequences of a launch: their stage prefix lives in LDS

// What a segment costs besides its steps (lengths, page ids, queries, the merge or the rows).  One
// tile, in stages of four steps: the bf16 rows at its kernel 92 us against 105 at 0.  More, in
// steps: 256 fp8 rows of 2,048 tokens at the median, 8 nodes, 492 us, 510 at 8, 530 at 4.
constexpr int kTreeNarrowCost = 2;
constexpr int kTreeWideCost = 12;

// Tiles of 32 columns (a node's query heads, node by node) of a workgroup, for `columns` =
// nodes x group.  28 columns in one tile 92 us, through LDS in two 114; 56 in two tiles 122, in four
// 130 (bf16; fp8, 32 and 64 columns: 371 and 431, 539 and 621; the rows are at the kernels).
inline int tree_tiles(int64_t columns) { return columns <= 32 ? 1 : columns <= 64 ? 2 : 4; }

struct TreeParams {
  const uint16_t* q;            // [B][T][Hq][d]
  const uint16_t* k_draft;      // [B][T][Hkv][d]
  const uint16_t* v_draft;
  const uint64_t* tree_mask;    // [B][T]
  const int32_t* node_counts;   // [B], or null: T
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  uint16_t* out;
  int4* cuts;                   // [workgroups] {b, head and column block, pieces, first slot}; b = -1: none
  float* part_o;                // [2 * workgroups][tiles][32 * d] partials, in the accumulators' lane order
  float2* part_ml;              // [2 * workgroups][tiles * 32] {max (log2 units), sum}
  int32_t num_seqs, num_nodes, num_q_heads, num_kv_heads, group, stride, blocks;
  int32_t whole;                // a workgroup per (sequence, KV head, column block); no cuts
  int64_t page_bytes;
  float scale_log2;
};

// One tile (tree_narrow.hip), or two or blocks of four (tree.hip).
hipError_t launch_tree_narrow(const TreeParams& p, int head_dim, int page_size, bool fp8,
                              int64_t grid, hipStream_t s);
hipError_t launch_tree_wide(const TreeParams& p, int head_dim, int page_size, bool fp8, int tiles,
                            int64_t grid, hipStream_t s);
hipError_t launch_tree_combine(const TreeParams& p, int head_dim, int tiles, int64_t grid,
                               hipStream_t s);

// Window attention.
struct WindowParams {
  const uint16_t* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  uint16_t* out;
  float* part_o;        // [segments * chunks][G][d] unnormalised partials
  float2* part_ml;      // {max (log2 units), sum}
  int64_t page_bytes;
  int32_t num_seqs, num_q_heads, num_kv_heads, group, stride, head_dim, page_size;
  int32_t window, sinks;
  int32_t chunk_pages;  // visible pages per workgroup
  int32_t chunks;       // workgroups per segment
  float scale_log2;
};

// The pages that a sequence of L tokens shows: the first `sink`, then first .. n - 1.
struct Visible {
  int n, sink, first;
  __host__ __device__ int pages() const { return sink + n - first; }
};
__host__ __device__ inline Visible visible_pages(int L, int P, int stride, int window, int sinks) {
  Visible v;
  if (L < 0) L = 0;
  const int64_t most = (int64_t)stride * P;
  if (L > most) L = (int)most;  // a contract violation stays in bounds
  v.n = (L + P - 1) / P;
  const int s = (int)(((int64_t)sinks + P - 1) / P);
  v.sink = s < v.n ? s : v.n;
  const int begin = L > window ? L - window : 0;
  v.first = begin / P > v.sink ? begin / P : v.sink;
  return v;
}

hipError_t launch_window(const WindowParams& p, bool fp8, hipStream_t s);
hipError_t launch_window_combine(const WindowParams& p, hipStream_t s);
hipError_t launch_window_validate(const ValidateParams& p, int window, int sinks, hipStream_t s);

// Path append.
struct PathParams {
  const uint16_t* k_new;       // bf16 [B][T][Hkv][d]
  const uint16_t* v_new;
  const int32_t* path;         // [B][T], or null: 0, 1, 2, ...
  const int32_t* counts;       // [B], or null: T
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* version_ids;  // ownership check when page_owner is set
  const int16_t* page_owner;
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;             // fp8 only
  float* v_scales;
  int32_t* dev_status;         // may be null
  int32_t num_seqs, num_tokens, num_kv_heads, head_dim, page_size, stride;
  int64_t num_pages;
};
hipError_t launch_append_path(const PathParams& p, bool fp8, hipStream_t s);

// Page copies.
struct CopyParams {
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
  const int32_t* src;
  const int32_t* dst;
  int32_t* dev_status;
  int64_t n_pages, num_pages, page_bytes;
  int32_t has_scales;
  int32_t layer;               // pages per grid layer, set by the launch
};
hipError_t launch_page_copy(const CopyParams& p, hipStream_t s);

}  // namespace dora
