// Internal declarations of attention over listed pages, the choice of pages and their
// bounds, and reads of the cache.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "cache_internal.h"
#include "dora.h"
#include "dora_internal.h"

namespace dora {

// Attention over listed pages.
struct PagesParams {
  const uint16_t* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* lists;   // [B][Hkv][list_stride], or null: all pages of a row
  const int32_t* counts;  // [B][Hkv]
  uint16_t* out;
  float* part_o;          // [segments * chunks][G][d] unnormalised partials
  float2* part_ml;        // {max (log2 units), sum}; max -inf: nothing attended
  int64_t page_bytes;
  int32_t num_seqs, num_q_heads, num_kv_heads, group, stride, head_dim, page_size;
  int32_t list_stride;
  int32_t chunk_pages;    // listed pages of a workgroup
  int32_t chunks;         // workgroups of a segment
  int32_t waves;          // of a workgroup: kSegWaves or 1
  float scale_log2;
};
hipError_t launch_pages(const PagesParams& p, int kv_dtype, hipStream_t s);
hipError_t launch_pages_combine(const PagesParams& p, hipStream_t s);
hipError_t launch_pages_validate(const ValidateParams& p, const int32_t* lists, const int32_t* counts,
                                 int num_kv_heads, int list_stride, hipStream_t s);

// Listed pages that a workgroup stages in LDS, at most.
constexpr int kPagesMaxChunk = 512;

struct PagesLayout {
  int chunk_pages, chunks;
  size_t part_o_off, part_ml_off, total;
};

// Listed pages of a workgroup, and what the workspace holds.
//   A list goes whole to one workgroup where it is short (768 tokens) or the segments are half
// as many as the CUs; fewer and longer ones are cut so that about 384 workgroups work, each of at
// least 128 tokens: a wave then still has one or two steps for its start and the combine.  Over
// 1,169 drawn batches (bf16, fp8 and 4-bit pages, lists of 128 to 8,192 tokens, up to 1,024 rows,
// counts full or uneven) this takes 1.03 of the time of the best power of two for each; at least
// 256 tokens and 1,024 workgroups, the rule before, 1.09 (512 lists of 2,048 tokens in bf16:
// 93.0 us by it, 86.5 whole; 3 lists of 2,000: 9.4 in chunks of 128, 10.5 of 256, 22.9 whole).
inline void pages_layout(const dora_decode_desc& d, int32_t list_stride, PagesLayout* w) {
  const int seqs = d.num_seqs < kMaxSeqsPerLaunch ? d.num_seqs : kMaxSeqsPerLaunch;
  const int64_t segs = (int64_t)seqs * d.num_kv_heads;
  int64_t chunk = list_stride;
  if (segs > 0 && segs < 128 && chunk * d.page_size > 768) {
    const int64_t parts = 384 / segs, least = 128 / d.page_size;
    chunk = ((chunk + parts - 1) / parts + least - 1) / least * least;
  }
  if (chunk > kPagesMaxChunk) chunk = kPagesMaxChunk;
  if (chunk > list_stride) chunk = list_stride;
  w->chunk_pages = (int)chunk;
  w->chunks = (int)((list_stride + chunk - 1) / chunk);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  const size_t slots = w->chunks > 1 ? (size_t)segs * w->chunks : 0;
  const size_t G = (size_t)(d.num_q_heads / d.num_kv_heads);
  w->part_o_off = kWsHeaderBytes;
  w->part_ml_off = up(w->part_o_off + slots * G * d.head_dim * 4);
  w->total = up(w->part_ml_off + slots * G * 8);
}

// Waves of a workgroup: four where a list is cut into chunks, else as many as a whole list of at most
// `tokens` wants.  With one, four times as many lists are
// under way and none is merged, but a list's steps follow each other: so for short lists of many
// segments, and of 4-bit pages (64 tokens a step) for all where the segments are two to a CU.
// Over 1,090 drawn batches of lists of 16 to 4,096 tokens this takes 1.01 of the better one's time,
// four waves always 1.16 for 4-bit pages, 1.07 for bf16 and 1.06 for fp8 (8,000 4-bit lists of 32
// tokens: 47 and 21 us; 1,024 of 2,560: 75.8 and 69.8; 4,000 fp8 lists of up to 3,200: 434 and 480).
inline int pages_waves(const dora_decode_desc& d, int chunks, int64_t segs, int64_t tokens) {
  if (chunks > 1) return kSegWaves;
  const bool one = d.kv_dtype == DORA_KV_FP4
                       ? (tokens <= 64 && segs >= 128) || (tokens <= 4096 && segs >= 512)
                       : (tokens <= 32 && segs >= 128) || (tokens <= 256 && segs >= 640);
  return one ? 1 : kSegWaves;
}

// The same for the 4-bit decode, whose rows (at most `tokens`, the table's width) are less even.
inline int pages4_waves(int64_t segs, int64_t tokens) {
  const bool one = (tokens <= 128 && segs >= 256) || (tokens <= 768 && segs >= 640) ||
                   (tokens <= 1536 && segs >= 2048);
  return one ? 1 : kSegWaves;
}

// Bytes of a page's bounds: int8 [Hkv][2][d] (largest, smallest), fp32 [Hkv] scales.
__host__ __device__ inline int64_t bounds_bytes(int64_t num_kv_heads, int64_t head_dim) {
  return (num_kv_heads * (2 * head_dim + 4) + 15) / 16 * 16;
}
// Bounds of the pages that the last tokens lie in (k_pages and k_scales are read).
hipError_t launch_page_bounds(const PathParams& p, const float* k_scales, uint8_t* bounds,
                              int kv_dtype, hipStream_t s);

struct SelectParams {
  const uint16_t* q;
  const uint8_t* bounds;
  const int32_t* block_table;
  const int32_t* seq_lens;
  float* scores;          // [B][Hkv][stride]
  int32_t* lists;         // [B][Hkv][budget]
  int32_t* counts;        // [B][Hkv]
  int64_t record;         // bytes of a page's bounds
  int32_t num_seqs, num_q_heads, num_kv_heads, group, stride, head_dim, page_size;
  int32_t budget, sinks, recent;
};
hipError_t launch_page_scores(const SelectParams& p, int cus, hipStream_t s);
hipError_t launch_page_select(const SelectParams& p, hipStream_t s);
// Whether one launch does both, and that launch (scores may be null then).
bool select_at_once(const SelectParams& p, int cus);
hipError_t launch_page_score_select(const SelectParams& p, hipStream_t s);

// Rows of the last tokens, as bf16 (PathParams' k_new, v_new and path are not used).
hipError_t launch_kv_read(const PathParams& p, const float* k_scales, const float* v_scales,
                          uint16_t* k_out, uint16_t* v_out, int kv_dtype, hipStream_t s);

}  // namespace dora
