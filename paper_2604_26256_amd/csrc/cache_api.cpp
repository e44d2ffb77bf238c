// C-ABI front end of the operators around the cache: tree and window attention, path
// append, page copies.  Argument validation (before any launch, no side effects),
// workspace layouts, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cache_internal.h"
#include "cache_rules.h"

using namespace dora;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

int compute_units() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus <= 0) {
    (void)hipGetLastError();  // no device here: size for a 256-CU part
    cus = 256;
  }
  return cus;
}

// The checks that both attention calls share, on a valid descriptor.
dora_status check_attn(const dora_decode_desc& d, const void* q, const void* k_pages,
                       const void* v_pages, const int32_t* block_table, const int32_t* seq_lens,
                       const int32_t* version_ids, const void* out, const void* workspace) {
  if (!q || !k_pages || !v_pages || !block_table || !seq_lens || !out || !workspace)
    return DORA_ERR_INVALID_ARG;
  if (d.kv_dtype == DORA_KV_FP8_E4M3 && (!d.k_scales || !d.v_scales)) return DORA_ERR_INVALID_ARG;
  if ((d.flags & DORA_FLAG_VALIDATE) && !version_ids && d.page_owner) return DORA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) ||
      !aligned16(workspace))
    return DORA_ERR_INVALID_ARG;
  return DORA_OK;
}

float scale_log2_of(const dora_decode_desc& d) {
  const float scale = d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim);
  // (the kernels take it for positive)
  return fmaxf(scale * 1.4426950408889634f, 1e-30f);
}

int64_t page_bytes_of(const dora_decode_desc& d) {
  return (int64_t)d.num_kv_heads * d.page_size * d.head_dim *
         (d.kv_dtype == DORA_KV_FP8_E4M3 ? 1 : 2);
}

dora_status check_nodes(int32_t num_nodes) {
  return num_nodes < 1 || num_nodes > 64 ? DORA_ERR_INVALID_ARG : DORA_OK;
}

dora_status check_window(int32_t window, int32_t sinks) {
  return window < 1 || sinks < 0 ? DORA_ERR_INVALID_ARG : DORA_OK;
}

dora_status validate_window(const dora_decode_desc& d, const int32_t* block_table,
                            const int32_t* seq_lens, const int32_t* version_ids, int32_t window,
                            int32_t sinks, int32_t* err, hipStream_t s) {
  if (launch_fill_i32(err, 0, 1, s) != hipSuccess) return DORA_ERR_HIP;
  ValidateParams vp{block_table, seq_lens, version_ids, d.page_owner, d.num_seqs,
                    d.page_size, d.block_table_stride, d.num_pages, err};
  if (launch_window_validate(vp, window, sinks, s) != hipSuccess) return DORA_ERR_HIP;
  int32_t host_err = 0;
  if (hipMemcpyAsync(&host_err, err, 4, hipMemcpyDeviceToHost, s) != hipSuccess ||
      hipStreamSynchronize(s) != hipSuccess)
    return DORA_ERR_HIP;
  return host_err ? DORA_ERR_DEVICE_CHECK : DORA_OK;
}

}  // namespace

extern "C" {

size_t dora_decode_tree_workspace_bytes(const dora_decode_desc* desc, int32_t num_nodes) {
  if (check_desc(desc) != DORA_OK || check_nodes(num_nodes) != DORA_OK) return 0;
  TreeLayout t;
  tree_layout(*desc, num_nodes, compute_units(), &t);
  return t.total;
}

dora_status dora_decode_attn_tree(const dora_decode_desc* desc, int32_t num_nodes, const void* q,
                                  const void* k_draft, const void* v_draft,
                                  const uint64_t* tree_mask, const int32_t* node_counts,
                                  const void* k_pages, const void* v_pages,
                                  const int32_t* block_table, const int32_t* seq_lens,
                                  const int32_t* version_ids, void* out, void* workspace,
                                  size_t workspace_bytes, dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_nodes(num_nodes);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  st = check_attn(d, q, k_pages, v_pages, block_table, seq_lens, version_ids, out, workspace);
  if (st != DORA_OK) return st;
  if (!k_draft || !v_draft || !tree_mask || !aligned16(k_draft) || !aligned16(v_draft))
    return DORA_ERR_INVALID_ARG;
  const int cus = compute_units();
  TreeLayout t;
  tree_layout(d, num_nodes, cus, &t);
  if (workspace_bytes < t.total) return DORA_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  uint8_t* ws = (uint8_t*)workspace;
  if (d.flags & DORA_FLAG_VALIDATE) {
    st = validate_tables(d, block_table, seq_lens, version_ids, (int32_t*)ws, s);
    if (st != DORA_OK) return st;
  }
  const bool fp8 = d.kv_dtype == DORA_KV_FP8_E4M3;
  for (int c0 = 0; c0 < d.num_seqs; c0 += t.seqs) {
    const int64_t nodes0 = (int64_t)c0 * num_nodes;  // node rows before this launch
    TreeParams p;
    p.q = (const uint16_t*)q + nodes0 * d.num_q_heads * d.head_dim;
    p.k_draft = (const uint16_t*)k_draft + nodes0 * d.num_kv_heads * d.head_dim;
    p.v_draft = (const uint16_t*)v_draft + nodes0 * d.num_kv_heads * d.head_dim;
    p.tree_mask = tree_mask + nodes0;
    p.node_counts = node_counts ? node_counts + c0 : nullptr;
    p.k_pages = (const uint8_t*)k_pages;
    p.v_pages = (const uint8_t*)v_pages;
    p.k_scales = d.k_scales;
    p.v_scales = d.v_scales;
    p.block_table = block_table + (int64_t)c0 * d.block_table_stride;
    p.seq_lens = seq_lens + c0;
    p.out = (uint16_t*)out + nodes0 * d.num_q_heads * d.head_dim;
    p.cuts = (int4*)(ws + t.cuts_off);
    p.part_o = (float*)(ws + t.part_o_off);
    p.part_ml = (float2*)(ws + t.part_ml_off);
    p.num_seqs = d.num_seqs - c0 < t.seqs ? d.num_seqs - c0 : t.seqs;
    p.num_nodes = num_nodes;
    p.num_q_heads = d.num_q_heads;
    p.num_kv_heads = d.num_kv_heads;
    p.group = d.num_q_heads / d.num_kv_heads;
    p.stride = d.block_table_stride;
    p.blocks = t.blocks;
    p.whole = tree_whole(d, t, p.num_seqs, cus) ? 1 : 0;
    p.page_bytes = page_bytes_of(d);
    p.scale_log2 = scale_log2_of(d);
    const int64_t grid =
        p.whole ? (int64_t)p.num_seqs * d.num_kv_heads * t.blocks : t.workgroups;
    const hipError_t e =
        t.tiles < 2 ? launch_tree_narrow(p, d.head_dim, d.page_size, fp8, grid, s)
                     : launch_tree_wide(p, d.head_dim, d.page_size, fp8, t.tiles, grid, s);
    if (e != hipSuccess) return DORA_ERR_HIP;
    if (!p.whole && launch_tree_combine(p, d.head_dim, t.tiles, grid, s) != hipSuccess)
      return DORA_ERR_HIP;
  }
  return DORA_OK;
}

size_t dora_decode_window_workspace_bytes(const dora_decode_desc* desc, int32_t window,
                                          int32_t sinks) {
  if (check_desc(desc) != DORA_OK || check_window(window, sinks) != DORA_OK) return 0;
  WindowLayout w;
  window_layout(*desc, window, sinks, &w);
  return w.total;
}

dora_status dora_decode_attn_window(const dora_decode_desc* desc, int32_t window, int32_t sinks,
                                    const void* q, const void* k_pages, const void* v_pages,
                                    const int32_t* block_table, const int32_t* seq_lens,
                                    const int32_t* version_ids, void* out, void* workspace,
                                    size_t workspace_bytes, dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  st = check_window(window, sinks);
  if (st != DORA_OK) return st;
  if (d.num_seqs == 0) return DORA_OK;
  st = check_attn(d, q, k_pages, v_pages, block_table, seq_lens, version_ids, out, workspace);
  if (st != DORA_OK) return st;
  WindowLayout w;
  window_layout(d, window, sinks, &w);
  if (workspace_bytes < w.total) return DORA_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t s = (hipStream_t)stream;
  uint8_t* ws = (uint8_t*)workspace;
  if (d.flags & DORA_FLAG_VALIDATE) {
    st = validate_window(d, block_table, seq_lens, version_ids, window, sinks, (int32_t*)ws, s);
    if (st != DORA_OK) return st;
  }
  const int64_t qrow = (int64_t)d.num_q_heads * d.head_dim;
  for (int c0 = 0; c0 < d.num_seqs; c0 += kMaxSeqsPerLaunch) {
    WindowParams p;
    p.q = (const uint16_t*)q + c0 * qrow;
    p.k_pages = (const uint8_t*)k_pages;
    p.v_pages = (const uint8_t*)v_pages;
    p.k_scales = d.k_scales;
    p.v_scales = d.v_scales;
    p.block_table = block_table + (int64_t)c0 * d.block_table_stride;
    p.seq_lens = seq_lens + c0;
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
    p.window = window;
    p.sinks = sinks;
    p.chunk_pages = w.chunk_pages;
    p.chunks = w.chunks;
    p.scale_log2 = scale_log2_of(d);
    if (launch_window(p, d.kv_dtype == DORA_KV_FP8_E4M3, s) != hipSuccess) return DORA_ERR_HIP;
    if (p.chunks > 1 && launch_window_combine(p, s) != hipSuccess) return DORA_ERR_HIP;
  }
  return DORA_OK;
}

dora_status dora_kv_append_path(const dora_decode_desc* desc, int32_t num_tokens,
                                const void* k_new, const void* v_new, const int32_t* path,
                                const int32_t* counts, const int32_t* block_table,
                                const int32_t* seq_lens, const int32_t* version_ids, void* k_pages,
                                void* v_pages, float* k_scales, float* v_scales,
                                int32_t* dev_status, dora_stream_t stream) {
  dora_status st = check_desc(desc);
  if (st != DORA_OK) return st;
  const dora_decode_desc& d = *desc;
  if (num_tokens < 1 || num_tokens > DORA_PATH_MAX_TOKENS) return DORA_ERR_INVALID_ARG;
  if (d.num_seqs == 0) return DORA_OK;
  const bool fp8 = d.kv_dtype == DORA_KV_FP8_E4M3;
  const bool validate = (d.flags & DORA_FLAG_VALIDATE) != 0;
  if (!k_new || !v_new || !block_table || !seq_lens || !k_pages || !v_pages)
    return DORA_ERR_INVALID_ARG;
  if (fp8 && (!k_scales || !v_scales)) return DORA_ERR_INVALID_ARG;
  if (validate && d.page_owner && !version_ids) return DORA_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pages) || !aligned16(v_pages))
    return DORA_ERR_INVALID_ARG;
  PathParams p;
  p.k_new = (const uint16_t*)k_new;
  p.v_new = (const uint16_t*)v_new;
  p.path = path;
  p.counts = counts;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.version_ids = validate ? version_ids : nullptr;
  p.page_owner = validate ? d.page_owner : nullptr;
  p.k_pages = (uint8_t*)k_pages;
  p.v_pages = (uint8_t*)v_pages;
  p.k_scales = fp8 ? k_scales : nullptr;
  p.v_scales = fp8 ? v_scales : nullptr;
  p.dev_status = dev_status;
  p.num_seqs = d.num_seqs;
  p.num_tokens = num_tokens;
  p.num_kv_heads = d.num_kv_heads;
  p.head_dim = d.head_dim;
  p.page_size = d.page_size;
  p.stride = d.block_table_stride;
  p.num_pages = d.num_pages;
  return launch_append_path(p, fp8, (hipStream_t)stream) == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}

dora_status dora_kv_page_copy(const dora_pack_desc* desc, void* k_pages, void* v_pages,
                              float* k_scales, float* v_scales, const int32_t* src_pages,
                              const int32_t* dst_pages, int64_t n_pages, int32_t* dev_status,
                              dora_stream_t stream) {
  dora_status st = check_pack_desc(desc);
  if (st != DORA_OK) return st;
  if (n_pages < 0 || n_pages > INT32_MAX) return DORA_ERR_INVALID_ARG;
  const bool fp8 = desc->kv_dtype == DORA_KV_FP8_E4M3;
  if (n_pages > 0) {
    if (!k_pages || !v_pages || !src_pages || !dst_pages) return DORA_ERR_INVALID_ARG;
    if (fp8 && (!k_scales || !v_scales)) return DORA_ERR_INVALID_ARG;
    if (!aligned16(k_pages) || !aligned16(v_pages)) return DORA_ERR_INVALID_ARG;
  }
  CopyParams p;
  p.k_pages = (uint8_t*)k_pages;
  p.v_pages = (uint8_t*)v_pages;
  p.k_scales = k_scales;
  p.v_scales = v_scales;
  p.src = src_pages;
  p.dst = dst_pages;
  p.dev_status = dev_status;
  p.n_pages = n_pages;
  p.num_pages = desc->num_pages;
  p.page_bytes = (int64_t)desc->num_kv_heads * desc->page_size * desc->head_dim * (fp8 ? 1 : 2);
  p.has_scales = fp8 ? 1 : 0;
  p.layer = 0;
  return launch_page_copy(p, (hipStream_t)stream) == hipSuccess ? DORA_OK : DORA_ERR_HIP;
}

}  // extern "C"
