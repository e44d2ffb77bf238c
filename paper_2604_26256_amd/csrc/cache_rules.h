// How the attention calls around the cache are launched and what their workspaces hold: column
// tiles, sequences of a launch, workgroups, whole rows or cut ones, pages of a workgroup.
// Host arithmetic on a valid descriptor and the device's compute units (cus).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "cache_internal.h"

namespace dora {

inline size_t ws_align(size_t x) { return (x + 255) / 256 * 256; }

// ---------------------------------------------------------------------------
// tree
// ---------------------------------------------------------------------------

struct TreeLayout {
  int tiles, blocks;   // column tiles of a workgroup, column blocks of a (sequence, KV head)
  int seqs;            // sequences of a launch
  int64_t workgroups;  // of a launch
  size_t cuts_off, part_o_off, part_ml_off, total;
};

inline void tree_layout(const dora_decode_desc& d, int32_t num_nodes, int cus, TreeLayout* t) {
  const int64_t columns = (int64_t)num_nodes * (d.num_q_heads / d.num_kv_heads);
  t->tiles = tree_tiles(columns);
  t->blocks = (int)((columns + 32 * t->tiles - 1) / (32 * t->tiles));
  // A launch's stages (steps, at most, and a segment's start) are counted in 32 bits, with room for
  // their rounding to ranges; one row's, of less than 2^19 pages, 128 heads and 9 blocks, always fit.
  const int64_t steps = ((int64_t)d.block_table_stride * d.page_size + 31) / 32 + 2 +
                        (kTreeWideCost > kTreeNarrowCost ? kTreeWideCost : kTreeNarrowCost);
  int64_t seqs = (INT32_MAX - 64) / (steps * d.num_kv_heads * t->blocks);
  if (seqs > kTreeMaxSeqs) seqs = kTreeMaxSeqs;
  t->seqs = (int)(seqs < d.num_seqs ? seqs : d.num_seqs);
  // Workgroups a CU.  One tile: two, but one where a wave holds two bf16 steps of 128 dims in
  // registers (92 us against 123 with half the registers).  Two tiles, of two waves: three (the 64
  // fp8 columns of 256 rows 500 us, 588 with two, 520 with four; bf16's LDS has no room for four).
  const bool large = d.head_dim == 128 && d.kv_dtype == DORA_KV_BF16;
  const int waves = t->tiles == 2 ? 2 : kTreeWaves;  // of a workgroup
  const int per_cu = t->tiles < 2 ? (large ? 1 : 2) : t->tiles == 2 ? 3 : 2;
  const int64_t slots = (int64_t)cus * per_cu;
  const int64_t most = (int64_t)t->seqs * d.num_kv_heads * t->blocks * steps;
  t->workgroups = d.num_waves > 0 ? ((int64_t)d.num_waves + waves - 1) / waves
                  : slots < most ? slots : most;
  if (t->workgroups < 1) t->workgroups = 1;
  size_t off = kWsHeaderBytes;
  t->cuts_off = off;
  off = ws_align(off + (size_t)t->workgroups * 16);
  t->part_o_off = off;
  off = ws_align(off + (size_t)(2 * t->workgroups) * t->tiles * 32 * d.head_dim * 4);
  t->part_ml_off = off;
  off = ws_align(off + (size_t)(2 * t->workgroups) * t->tiles * 32 * 8);
  t->total = off;
}

// Whether a launch takes a workgroup per (sequence, KV head, column block), uncut: where no row
// is longer than 2,048 tokens and, with more than one tile (whose workgroups take all of a row's
// steps one by one), the workgroups fill the chip or no row passes 512.  Against equal ranges and
// their join: one tile, 128 fp8 rows of 400 tokens at the median, 8 heads of 128, 43 us for 53, 8 bf16 rows
// of 1,024, 2 heads of 64, 10.2 for 12.5, of 4,096, 23 for 17; two tiles, 256 bf16 rows of up to
// 1,024, 4 heads, 60 for 67, 64 of 2,048, 62 for 76, but 4 fp8 rows of 1,024, 8 heads, 30 for 25, of
// 2,048, 52 for 31.
inline bool tree_whole(const dora_decode_desc& d, const TreeLayout& t, int seqs, int cus) {
  const int64_t tokens = (int64_t)d.block_table_stride * d.page_size;
  const int64_t groups = (int64_t)seqs * d.num_kv_heads * t.blocks;
  return d.num_waves <= 0 &&
         (tokens <= 512 || (tokens <= 2048 && (t.tiles < 2 || groups >= cus)));
}

// ---------------------------------------------------------------------------
// window
// ---------------------------------------------------------------------------

struct WindowLayout {
  int chunk_pages, chunks;
  size_t part_o_off, part_ml_off, total;
};

// Pages that a sequence can show, at most.
inline int64_t most_visible(const dora_decode_desc& d, int32_t window, int32_t sinks) {
  const int64_t P = d.page_size;
  const int64_t n = (window + P - 2) / P + 1 + (sinks + P - 1) / P;
  return n < d.block_table_stride ? n : d.block_table_stride;
}

inline void window_layout(const dora_decode_desc& d, int32_t window, int32_t sinks, WindowLayout* w) {
  const int64_t most = most_visible(d, window, sinks);
  const int seqs = d.num_seqs < kMaxSeqsPerLaunch ? d.num_seqs : kMaxSeqsPerLaunch;
  const int64_t segs = (int64_t)seqs * d.num_kv_heads;
  int64_t chunk = segs > 0 ? (most * segs + 1023) / 1024 : most;  // about 1,024 workgroups
  const int64_t least = 256 / d.page_size;
  chunk = (chunk + least - 1) / least * least;
  // A lane holds each page of its wave.  What a window has beyond 256 pages, be it one, is a part of
  // its own: level with equal parts (128 rows of 8,000 tokens through 4,096, 8 heads of 128, pages of
  // 16: bf16 345 us, 351 in equal parts, fp8 206 and 211) or faster (400 rows, fp8, 612 and 642), as the
  // few short workgroups run beside the rest, and rows of 130 to 256 pages stay whole.
  if (chunk > 64 * kSegWaves) chunk = 64 * kSegWaves;
  if (chunk > most) chunk = most;
  w->chunk_pages = (int)chunk;
  w->chunks = (int)((most + chunk - 1) / chunk);
  size_t off = kWsHeaderBytes;
  const size_t slots = w->chunks > 1 ? (size_t)segs * w->chunks : 0;
  const size_t G = (size_t)(d.num_q_heads / d.num_kv_heads);
  w->part_o_off = off;
  off = ws_align(off + slots * G * d.head_dim * 4);
  w->part_ml_off = off;
  off = ws_align(off + slots * G * 8);
  w->total = off;
}

}  // namespace dora
