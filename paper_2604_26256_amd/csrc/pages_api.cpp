// C-ABI front end of the operators that read less of the cache: attention over listed pages,
// their choice and bounds, and reads of the last rows.  Argument validation (before any launch,
// no side effects), workspace layouts, launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "api_checks.h"
#include "pages_internal.h"

using namespace dora;

namespace {

dora_status check_lists(int32_t list_stride) {
  return list_stride < 1 || list_stride >= (1 << 19) ? DORA_ERR_INVALID_ARG : DORA_OK;
}

dora_status check_select(int32_t budget, int32_t sink_pages, int32_t recent_pages) {
  if (check_lists(budget) != DORA_OK || sink_pages < 0 || recent_pages < 0 ||
      (int64_t)sink_pages + recent_pages > budget)
    return DORA_ERR_INVALID_ARG;
  return DORA_OK;
}

dora_status validate_lists(const dora_decode_desc& d, int32_t list_stride, const int32_t* lists,
                           const int32_t* counts, const int32_t* block_table, const int32_t* seq_lens,
                           const int32_t* version_ids, int32_t* err, hipStream_t s) {
  if (launch_fill_i32(err, 0, 1, s) != hipSuccess) return DORA_ERR_HIP;
  for (int c0 = 0; c0 < d.num_seqs; c0 += kMaxSeqsPerLaunch) {
    const int seqs = d.num_seqs - c0 < kMaxSeqsPerLaunch ? d.num_seqs - c0 : kMaxSeqsPerLaunch;
    const int64_t seg0 = (int64_t)c0 * d.num_kv_heads;
    ValidateParams vp{block_table + (int64_t)c0 * d.block_table_stride,
                      seq_lens + c0,
                      version_ids ? version_ids + c0 : nullptr,
                      d.page_owner,
                      seqs,
                      d.page_size,
                      d.block_table_stride,
                      d.num_pages,
                      err};
    if (launch_pages_validate(vp, lists + seg0 * list_stride, counts + seg0, d.num_kv_heads,
                              list_stride, s) != hipSuccess)
      return DORA_ERR_HIP;
  }
  int32_t host_err = 0;
  if (hipMemcpyAsync(&host_err, err, 4, hipMemcpyDeviceToHost, s) != hipSuccess ||
      hipStreamSynchronize(s) != hipSuccess)
    return DORA_ERR_HIP;
  return host_err ? DORA_ERR_DEVICE_CHECK : DORA_OK;
}

// The last tokens of each sequence, for the calls that go by them.
PathParams last_tokens(const dora_decode_desc& d, int32_t num_tokens, const int32_t* counts,
                       const int32_t* block_table, const int32_t* seq_lens,
                       const int32_t* version_ids, int32_t* dev_status) {
  const bool validate = (d.flags & DORA_FLAG_VALIDATE) != 0;
  PathParams p{};
  p.counts = counts;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.version_ids = validate ? version_ids : nullptr;
  p.page_owner = validate ? d.page_owner : nullptr;
  p.dev_status = dev_status;
  p.num_seqs = d.num_seqs;
  p.num_tokens = num_tokens;
  p.num_kv_heads = d.num_kv_heads;
  p.head_dim = d.head_dim;
  p.page_size = d.page_size;
  p.stride = d.block_table_stride;
  p.num_pages = d.num_pages;
  return p;
}

dora_status check_last(int32_t num_tokens) {
  return num_tokens < 1 || num_tokens > DORA_PATH_MAX_TOKENS ? DORA_ERR_INVALID_ARG : DORA_OK;
}

}  // namespace

extern "C" {

size_t dora_decode_pages_workspace_bytes(const dora_decode_desc* desc, int32_t list_stride) {
  if (check_desc(desc) != DORA_OK || check_lists(list_stride) != DORA_OK) return 0;
  PagesLayout w;
  pages_layout(*desc, list_stride, &w);
  return w.total;
}

dora_status dora_decode_attn_pages(const dora_decode_desc* desc, int32_t list_stride, const void* q,
                                   const int32_t* page_lists, const int32_t* page_counts,
                                   const void* k_pages, const void* v_pages,
                                   const int32_t* block_table, const int32_t* seq_lens,
                                   const int32_t* version_ids, void* out, void* workspace,
                                   size_t workspace_bytes, dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_lists(list_stride);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  st = check_attn(d, q, k_pages, v_pages, block_table, seq_lens, version_ids, out, workspace);
  if (st != DORA_OK) return st;
  if (!page_lists || !page_counts) return DORA_ERR_INVALID_ARG;
  PagesLayout w;
  pages_layout(d, list_stride, &w);
  if (workspace_bytes < w.total) return DORA_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  uint8_t* ws = (uint8_t*)workspace;
  if (d.flags & DORA_FLAG_VALIDATE) {
    st = validate_lists(d, list_stride, page_lists, page_counts, block_table, seq_lens, version_ids,
                        (int32_t*)ws, s);
    if (st != DORA_OK) return st;
  }
  const int64_t qrow = (int64_t)d.num_q_heads * d.head_dim;
  for (int c0 = 0; c0 < d.num_seqs; c0 += kMaxSeqsPerLaunch) {
    const int64_t seg0 = (int64_t)c0 * d.num_kv_heads;
    PagesParams p;
    p.q = (const uint16_t*)q + c0 * qrow;
    p.k_pages = (const uint8_t*)k_pages;
    p.v_pages = (const uint8_t*)v_pages;
    p.k_scales = d.k_scales;
    p.v_scales = d.v_scales;
    p.block_table = block_table + (int64_t)c0 * d.block_table_stride;
    p.seq_lens = seq_lens + c0;
    p.lists = page_lists + seg0 * list_stride;
    p.counts = page_counts + seg0;
    p.out = (uint16_t*)out + c0 * qrow;
    p.part_o = (float*)(ws + w.part_o_off);
    p.part_ml = (float2*)(ws + w.part_ml_off);
    p.page_bytes = page_bytes_of(d);
    p.num_seqs = d.num_seqs - c0 < kMaxSeqsPerLaunch ? d.num_seqs - c0 : kMaxSeqsPerLaunch;
    p.num_q_heads = d.num_q_heads;
    p.num_kv_heads = d.num_kv_heads;
    p.group = d.num_q_heads / d.num_kv_heads;
    p.stride = d.block_table_stride;
    p.head_dim = d.head_dim;
    p.page_size = d.page_size;
    p.list_stride = list_stride;
    p.chunk_pages = w.chunk_pages;
    p.chunks = w.chunks;
    p.waves = pages_waves(d, w.chunks, (int64_t)p.num_seqs * d.num_kv_heads,
                          (int64_t)list_stride * d.page_size);
    p.scale_log2 = scale_log2_of(d);
    if (launch_pages(p, d.kv_dtype, s) != hipSuccess) return DORA_ERR_HIP;
    if (p.chunks > 1 && launch_pages_combine(p, s) != hipSuccess) return DORA_ERR_HIP;
  }
  return DORA_OK;
}

size_t dora_page_bounds_bytes(int32_t num_kv_heads, int32_t head_dim) {
  if (num_kv_heads < 1 || num_kv_heads > 127 || (head_dim != 64 && head_dim != 128)) return 0;
  return (size_t)bounds_bytes(num_kv_heads, head_dim);
}

dora_status dora_kv_page_bounds(const dora_decode_desc* desc, int32_t num_tokens,
                                const int32_t* counts, const void* k_pages,
                                const int32_t* block_table, const int32_t* seq_lens,
                                const int32_t* version_ids, void* bounds, int32_t* dev_status,
                                dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_last(num_tokens);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  if (!k_pages || !block_table || !seq_lens || !bounds) return DORA_ERR_INVALID_ARG;
  if (d.kv_dtype == DORA_KV_FP8_E4M3 && !d.k_scales) return DORA_ERR_INVALID_ARG;
  if ((d.flags & DORA_FLAG_VALIDATE) && d.page_owner && !version_ids) return DORA_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(bounds)) return DORA_ERR_INVALID_ARG;
  PathParams p = last_tokens(d, num_tokens, counts, block_table, seq_lens, version_ids, dev_status);
  p.k_pages = (uint8_t*)k_pages;  // (read only)
  return launch_page_bounds(p, d.k_scales, (uint8_t*)bounds, d.kv_dtype, (hipStream_t)stream) ==
                 hipSuccess
             ? DORA_OK
             : DORA_ERR_HIP;
}

size_t dora_page_select_workspace_bytes(const dora_decode_desc* desc) {
  if (check_desc(desc) != DORA_OK) return 0;
  const int seqs = desc->num_seqs < kMaxSeqsPerLaunch ? desc->num_seqs : kMaxSeqsPerLaunch;
  return kWsHeaderBytes + (size_t)seqs * desc->num_kv_heads * desc->block_table_stride * 4;
}

dora_status dora_page_select(const dora_decode_desc* desc, int32_t budget, int32_t sink_pages,
                             int32_t recent_pages, const void* q, const void* bounds,
                             const int32_t* block_table, const int32_t* seq_lens,
                             const int32_t* version_ids, int32_t* page_lists, int32_t* page_counts,
                             float* scores, void* workspace, size_t workspace_bytes,
                             dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_select(budget, sink_pages, recent_pages);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  if (!q || !bounds || !block_table || !seq_lens || !page_lists || !page_counts || !workspace)
    return DORA_ERR_INVALID_ARG;
  if ((d.flags & DORA_FLAG_VALIDATE) && !version_ids && d.page_owner) return DORA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(bounds) || !aligned16(workspace)) return DORA_ERR_INVALID_ARG;
  if (workspace_bytes < (scores ? kWsHeaderBytes : dora_page_select_workspace_bytes(desc)))
    return DORA_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  uint8_t* ws = (uint8_t*)workspace;
  if (d.flags & DORA_FLAG_VALIDATE) {
    st = validate_tables(d, block_table, seq_lens, version_ids, (int32_t*)ws, s);
    if (st != DORA_OK) return st;
  }
  const int cus = compute_units();
  for (int c0 = 0; c0 < d.num_seqs; c0 += kMaxSeqsPerLaunch) {
    const int64_t seg0 = (int64_t)c0 * d.num_kv_heads;
    SelectParams p;
    p.q = (const uint16_t*)q + (int64_t)c0 * d.num_q_heads * d.head_dim;
    p.bounds = (const uint8_t*)bounds;
    p.block_table = block_table + (int64_t)c0 * d.block_table_stride;
    p.seq_lens = seq_lens + c0;
    p.scores = scores ? scores + seg0 * d.block_table_stride : (float*)(ws + kWsHeaderBytes);
    p.lists = page_lists + seg0 * budget;
    p.counts = page_counts + seg0;
    p.record = bounds_bytes(d.num_kv_heads, d.head_dim);
    p.num_seqs = d.num_seqs - c0 < kMaxSeqsPerLaunch ? d.num_seqs - c0 : kMaxSeqsPerLaunch;
    p.num_q_heads = d.num_q_heads;
    p.num_kv_heads = d.num_kv_heads;
    p.group = d.num_q_heads / d.num_kv_heads;
    p.stride = d.block_table_stride;
    p.head_dim = d.head_dim;
    p.page_size = d.page_size;
    p.budget = budget;
    p.sinks = sink_pages;
    p.recent = recent_pages;
    if (select_at_once(p, cus)) {
      p.scores = scores ? p.scores : nullptr;
      if (launch_page_score_select(p, s) != hipSuccess) return DORA_ERR_HIP;
      continue;
    }
    if (launch_page_scores(p, cus, s) != hipSuccess) return DORA_ERR_HIP;
    if (launch_page_select(p, s) != hipSuccess) return DORA_ERR_HIP;
  }
  return DORA_OK;
}

dora_status dora_kv_read(const dora_decode_desc* desc, int32_t num_tokens, const int32_t* counts,
                         const void* k_pages, const void* v_pages, const int32_t* block_table,
                         const int32_t* seq_lens, const int32_t* version_ids, void* k_out, void* v_out,
                         int32_t* dev_status, dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_last(num_tokens);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  if (!k_pages || !v_pages || !block_table || !seq_lens || !k_out || !v_out)
    return DORA_ERR_INVALID_ARG;
  if (d.kv_dtype == DORA_KV_FP8_E4M3 && (!d.k_scales || !d.v_scales)) return DORA_ERR_INVALID_ARG;
  if ((d.flags & DORA_FLAG_VALIDATE) && d.page_owner && !version_ids) return DORA_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_out) || !aligned16(v_out))
    return DORA_ERR_INVALID_ARG;
  PathParams p = last_tokens(d, num_tokens, counts, block_table, seq_lens, version_ids, dev_status);
  p.k_pages = (uint8_t*)k_pages;  // (read only)
  p.v_pages = (uint8_t*)v_pages;
  const bool fp8 = d.kv_dtype == DORA_KV_FP8_E4M3;
  return launch_kv_read(p, fp8 ? d.k_scales : nullptr, fp8 ? d.v_scales : nullptr, (uint16_t*)k_out,
                        (uint16_t*)v_out, d.kv_dtype, (hipStream_t)stream) == hipSuccess
             ? DORA_OK
             : DORA_ERR_HIP;
}

}  // extern "C"
