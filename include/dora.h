/*
 * dora.h — C ABI of the MI355X (gfx950) decode-attention hot path of DORA's
 * rollout stage ("DORA: A Scalable Asynchronous Reinforcement Learning System
 * for Language Model Training", arXiv 2604.26256).
 *
 * What the paper fixes and this library implements:
 *   - Rollout decode is memory-bound and dominates the RL step (Sec. 1;
 *     Sec. 2.2, Eq. (1) and the TPOT term tau in it).  Each decode step attends
 *     every active sequence's cached keys and values; response lengths are
 *     heavily long-tailed (Sec. 2.2, "Workload skewness").
 *   - Sequences of several policy versions coexist in one rollout instance;
 *     every request carries the version tag it was dispatched under (Sec. 3.2,
 *     "Multi-version policy management").  Here: one shared page pool, one
 *     block-table row per sequence, and version_ids[b] per sequence.
 *   - KV states of a trajectory are identical on every instance that hosts its
 *     version, so migration moves the KV pages instead of re-running prefill
 *     (Sec. 3.4, "KV-Cache Reuse", two-phase state transfer).  Here: the page
 *     gather/scatter dora_kv_page_pack / dora_kv_page_unpack, bit-exact.
 *
 * Conventions shared by every entry point:
 *   - Every pointer named "device" is a HIP device pointer owned by the caller.
 *     The library never allocates, frees or retains device memory.
 *   - Every device-side entry point enqueues work on `stream` and returns
 *     without synchronising (graph-capturable), except where a flag says so.
 *   - All host-checkable errors (null pointers, unsupported shapes, a too-small
 *     workspace or packed buffer, version mismatch) are reported BEFORE any
 *     launch and leave every buffer untouched.  Nothing throws or aborts across
 *     this ABI.  Device-data errors (a page id outside the pool, a page not
 *     owned by the sequence's version, seq_lens[b] > block_table_stride *
 *     page_size) are undefined behaviour unless DORA_FLAG_VALIDATE is set.
 *   - No global mutable state, with one exception: the fixed per-GPU
 *     workspace of dora_decode_attn_noalloc (calls of that entry point that
 *     overlap on one GPU race on it).  Pool objects are single-threaded.
 *
 * Data layouts (row-major, innermost index last; e = 2 bytes for bf16, 1 for
 * fp8; X = 16 / e, i.e. one 16-byte chunk of the head dimension):
 *   q, out       [num_seqs][num_q_heads][head_dim]                       bf16
 *   k_pages      [num_pages][num_kv_heads][head_dim / X][page_size][X]   bf16 | fp8
 *                (each token's key is cut into 16-byte chunks; chunk c of all
 *                 page_size tokens is stored contiguously)
 *   v_pages      [num_pages][num_kv_heads][head_dim][page_size]          bf16 | fp8
 *                (values stored transposed: the page_size tokens of one
 *                 head-dim index are contiguous)
 *   k_scales, v_scales  [num_pages] fp32 (fp8 only): stored value times the
 *                page's scale is the key/value (one scale per page, shared by
 *                all heads and tokens of that page)
 *   4-bit pages (DORA_KV_FP4): k_pages, v_pages [num_pages][num_kv_heads] tiles of
 *                page_size * head_dim * 17 / 32 bytes, scales among them:
 *                K  E2M1 codes [head_dim / 32][page_size][32], two in a byte (the
 *                   even one in its low half), then for each 32 dims of a token
 *                   the exponent, biased by 127, of the power of two that the
 *                   codes are times: bytes [head_dim / 32][page_size / 16][4][4],
 *                   that of slot 16 a + 4 b + c at [a][c][b]; 255 stands for NaN
 *                V  E2M1 codes [head_dim][page_size], two in a byte, then a bf16
 *                   scale for each 64 dims of a token [head_dim / 64][page_size]
 *                (attention over pages of 32 tokens takes 6 to 20 % less time than over
 *                 pages of 16, whose tiles are 8.5 lines of memory, or 4.25)
 *   block_table  [num_seqs][block_table_stride] int32 page ids, logical order
 *   seq_lens     [num_seqs] int32, tokens to attend (>= 0)
 *   version_ids  [num_seqs] int32 policy version of each sequence
 * fp8 is OCP E4M3FN (bias 7, max 448, S.1111.111 = NaN, no infinity).  E2M1 codes
 * stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6 and, with bit 3 set, their negatives.
 * GQA mapping: query head h reads KV head h / (num_q_heads / num_kv_heads).
 * Slots of the last page beyond seq_lens[b] are never used in the arithmetic
 * (they may hold any bytes, NaN included).
 *
 * The operation (dora_decode_attn), for every sequence b and query head h,
 * with G = num_q_heads / num_kv_heads, g = h / G, L = seq_lens[b]:
 *   K_t, V_t = key/value of token t < L, read from page block_table[b][t / P]
 *              at slot t % P, KV head g (times the page scale for fp8)
 *   s_t      = sm_scale * <q[b][h], K_t>
 *   out[b][h] = sum_t exp(s_t - max s) V_t / sum_t exp(s_t - max s)
 *   L = 0 gives out[b][h] = 0.
 */
#ifndef DORA_H
#define DORA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Opaque stream handle: a hipStream_t (NULL = the legacy default stream). */
typedef void* dora_stream_t;

typedef enum {
  DORA_OK = 0,
  DORA_ERR_INVALID_ARG = 1,          /* null pointer, bad count or bad geometry */
  DORA_ERR_UNSUPPORTED = 2,          /* head_dim / page_size / group size / dtype not built */
  DORA_ERR_WORKSPACE_TOO_SMALL = 3,  /* workspace or packed buffer smaller than required */
  DORA_ERR_VERSION_MISMATCH = 4,     /* pages of one policy version sent to another */
  DORA_ERR_POOL_EXHAUSTED = 5,       /* pool has too few free pages (state unchanged) */
  DORA_ERR_DEVICE_CHECK = 6,         /* DORA_FLAG_VALIDATE found bad device data */
  DORA_ERR_HIP = 7,                  /* a HIP runtime call failed */
  DORA_ERR_NOT_FOUND = 8             /* unknown sequence id in a pool call */
} dora_status;

typedef enum {
  DORA_KV_BF16 = 0,
  DORA_KV_FP8_E4M3 = 1,
  DORA_KV_FP4 = 4            /* E2M1 codes with scales in the pages; tree, window and
                                grouped attention are not built for it */
} dora_kv_dtype;

/* Flags for dora_decode_desc.flags. */
#define DORA_FLAG_VALIDATE    0x1u  /* range- and ownership-check every page id read;
                                       synchronises the stream and returns
                                       DORA_ERR_DEVICE_CHECK on bad device data */

/* Geometry and options of one decode-attention call.  Supported builds:
 * head_dim in {64, 128}; page_size in {16, 32}; group size num_q_heads /
 * num_kv_heads in [1, 16]; kv_dtype bf16, fp8 e4m3 or 4-bit (where a call does not
 * say otherwise). */
typedef struct {
  int32_t num_seqs;            /* B >= 0 */
  int32_t num_q_heads;         /* Hq, multiple of num_kv_heads */
  int32_t num_kv_heads;        /* Hkv >= 1 */
  int32_t head_dim;            /* d */
  int32_t page_size;           /* P tokens per page */
  int32_t block_table_stride;  /* int32 entries per block-table row (>= 1) */
  int64_t num_pages;           /* pool capacity in pages (for VALIDATE range checks) */
  int32_t kv_dtype;            /* dora_kv_dtype */
  float   sm_scale;            /* softmax scale; 0 means 1/sqrt(head_dim) */
  const float* k_scales;       /* device [num_pages] fp32, fp8 only (else NULL) */
  const float* v_scales;       /* device [num_pages] fp32, fp8 only (else NULL) */
  const int16_t* page_owner;   /* device [num_pages] owning version, or NULL; read
                                  only under DORA_FLAG_VALIDATE */
  uint32_t flags;              /* DORA_FLAG_* */
  int32_t num_waves;           /* decode wavefronts to launch; 0 = library
                                  default: per compute unit of the current
                                  device at most 4 for bf16 and 4-bit pages
                                  and 7 for fp8 pages, within the resident
                                  wavefront slots; never more than the batch
                                  can use
                                  (B x Hkv x stride page-heads over the minimum
                                  range).  With both this and min_range_pages 0,
                                  batches whose block tables are short or few
                                  are cut per segment instead (see
                                  dora_decode_attn) */
  int32_t min_range_pages;     /* smallest work range per wavefront, in
                                  (page, KV head) units, of 4-bit pages in (64
                                  tokens, KV head); 0 = library default */
} dora_decode_desc;

/* Human-readable name of a status code (static storage); "unknown status" for
 * a value that is no dora_status.  The code is passed as an int, so any value
 * is a valid argument. */
const char* dora_status_string(int status);

/* Bytes of device workspace dora_decode_attn needs for this geometry on the
 * current device (valid for every seq_lens the call may see).  Returns 0 for an
 * invalid or unsupported descriptor.  The workspace holds a 256-byte flag
 * header, one cut record per decode wavefront (or per (sequence, KV head)
 * segment, when there are no more segments than wavefronts) and two partial
 * results per wavefront (unnormalised output, running max and sum in fp32);
 * the batch's page prefix is built in each wavefront's LDS. */
size_t dora_decode_workspace_bytes(const dora_decode_desc* desc);

/* Decode wavefronts dora_decode_attn launches per launch for this descriptor on
 * the current device: desc->num_waves when it is set, else the library default
 * described at dora_decode_desc.num_waves.  Wavefront w takes page-heads
 * [w*T/W', (w+1)*T/W') of the launch's T (sequence, KV head, page) work items
 * in (sequence, head, page) order, where W' = min(W, ceil(T / m)), m being
 * desc->min_range_pages or 8 when that is 0, and the first T mod W' ranges hold
 * one extra item; so a caller can tell which (sequence, KV head) segments a
 * call cuts across wavefronts (except batches cut per segment, see
 * dora_decode_attn).  Of 4-bit pages the work items are steps of 64 tokens, and
 * m is 4 where min_range_pages is 0.  Each launch covers at most 8192 sequences.
 * Returns 0 for an invalid or unsupported descriptor. */
int64_t dora_decode_num_waves(const dora_decode_desc* desc);

/* Decode-step attention over the paged, multi-version KV pool (the operation
 * defined at the top of this file; the step the paper times as tau per output
 * token, Sec. 2.2 Eq. (1); version tags per Sec. 3.2).
 *   q            device bf16 [B][Hq][d]
 *   k_pages      device, layout above
 *   v_pages      device, layout above
 *   block_table  device int32 [B][block_table_stride]
 *   seq_lens     device int32 [B]
 *   version_ids  device int32 [B]; does not enter the arithmetic.  Under
 *                DORA_FLAG_VALIDATE every page b reads must satisfy
 *                page_owner[page] == version_ids[b].  May be NULL without it.
 *   out          device bf16 [B][Hq][d], written for every (b, h)
 *   workspace    device, >= dora_decode_workspace_bytes(desc) bytes, 16-byte
 *                aligned; contents on entry are ignored
 * Launches the decode kernel and a log-sum-exp combine kernel on `stream` (per
 * 8192 sequences).  Every decode wavefront takes an equal share of the batch's
 * (page, KV head) work, whatever the length mix.  Batches with few (sequence, KV
 * head) segments or short block tables run per segment instead, by lines on both
 * and on the page geometry: one workgroup per segment, in one launch (rows of up to
 * 512-2,048 tokens), or one per chunk of 256 or 512 tokens of it and a combine (rows
 * from 768 tokens on); dora_decode_segment_pages in dora_measure.h tells which.
 * Results do not depend on the number of wavefronts beyond fp32 rounding, and
 * repeated calls on the same inputs and device are bitwise identical.
 * Scores and sums are held in fp32.  Of 4-bit pages values of up to 2^127 give a finite
 * result; of bf16 and fp8 pages the magnitudes of the values that a row attends, each
 * times its weight relative to the row's largest, have to add up to less than 2^128. */
dora_status dora_decode_attn(const dora_decode_desc* desc,
                             const void* q, const void* k_pages, const void* v_pages,
                             const int32_t* block_table, const int32_t* seq_lens,
                             const int32_t* version_ids, void* out,
                             void* workspace, size_t workspace_bytes,
                             dora_stream_t stream);

/* Size of the fixed device array dora_decode_attn_noalloc uses as its
 * workspace, one per GPU. */
#define DORA_NOALLOC_WORKSPACE_BYTES ((size_t)48 << 20)

/* dora_decode_attn for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.
 * Same arguments, results and errors as dora_decode_attn, without the
 * workspace: the call uses a fixed array of DORA_NOALLOC_WORKSPACE_BYTES in
 * device memory that the library holds on each GPU it runs on, from load until
 * the process ends.  It allocates and frees nothing; its first call on a device
 * looks the array's address up.
 *   DORA_ERR_WORKSPACE_TOO_SMALL  dora_decode_workspace_bytes(desc) exceeds the
 *                                 array (e.g. a large desc->num_waves)
 *   DORA_ERR_INVALID_ARG          DORA_FLAG_VALIDATE set (it synchronises and
 *                                 copies to the host); plus dora_decode_attn's
 * Every call on one GPU uses that GPU's array, and the array keeps the last
 * call's contents (the decode ignores them): calls that overlap on one GPU (on
 * different streams or from different threads) race, and the caller must
 * order them. */
dora_status dora_decode_attn_noalloc(const dora_decode_desc* desc,
                                     const void* q, const void* k_pages, const void* v_pages,
                                     const int32_t* block_table, const int32_t* seq_lens,
                                     const int32_t* version_ids, void* out,
                                     dora_stream_t stream);

/* Decode attention for a batch made of response groups that share a prompt
 * (the responses sampled per prompt for GRPO-style advantages, App. B).  The
 * result equals dora_decode_attn's on the same arguments (up to fp32 rounding);
 * what changes is that each group's shared prompt pages are read from HBM once
 * instead of once per member.
 *   group_size    M >= 1; sequences [k*M, (k+1)*M) form group k; num_seqs must
 *                 be a multiple of M; M * (num_q_heads / num_kv_heads) <= 128
 *                 (else DORA_ERR_UNSUPPORTED)
 *   shared_pages_out  device int32 [num_seqs / M] or NULL: receives each
 *                 group's shared prefix S_k (below)
 *   other arguments as for dora_decode_attn; the workspace must hold
 *   dora_decode_grouped_workspace_bytes(desc, group_size) bytes.
 * Sharing is read off the block tables on the device: S_k is the number of
 * leading pages that every member of group k holds in full (j < seq_len /
 * page_size) under the same page id as the group's first member; a group of
 * one shares nothing.  Any batch is valid input (S_k = 0 where nothing is
 * shared).  Steps, all enqueued on `stream`, no host round trip: a prefix
 * kernel (per group, KV head and chunk of shared pages: finds S_k, reads the
 * pages once and applies them to every member's query heads); the
 * ordinary decode over each member's remaining pages; its combine, which
 * merges cut segments and folds every row with its group's prefix into out.
 * With shared_pages_out NULL, batches that dora_decode_attn cuts per segment
 * (small ones) run as that call does: it is faster there. */
size_t dora_decode_grouped_workspace_bytes(const dora_decode_desc* desc, int32_t group_size);
dora_status dora_decode_attn_grouped(const dora_decode_desc* desc, const void* q,
                                     const void* k_pages, const void* v_pages,
                                     const int32_t* block_table, const int32_t* seq_lens,
                                     const int32_t* version_ids, void* out, int32_t group_size,
                                     int32_t* shared_pages_out, void* workspace,
                                     size_t workspace_bytes, dora_stream_t stream);

/* Decode attention for a tree of drafted tokens per sequence (verification of
 * speculative drafts): num_nodes query rows of a sequence share one pass over its
 * cached tokens.  With T = num_nodes, n = node_counts[b] (T without node_counts) and
 * L = seq_lens[b], for every node i < n and query head h, g = h / G:
 *   s_t   = sm_scale * <q[b][i][h], K_t>              t < L (the cache, as above)
 *   s'_j  = sm_scale * <q[b][i][h], k_draft[b][j][g]>  j < n with bit j of
 *                                                     tree_mask[b][i] set
 *   out[b][i][h] = softmax over all of them, applied to V_t and v_draft[b][j][g]
 * A node that sees nothing (L = 0 and no bit) gives 0; rows of nodes i >= n are left
 * as they were.  The mask is taken as it is: a node that attends itself has its own
 * bit set, and bits of nodes >= n count as 0.  What a draft holds, infinities and NaN
 * too, reaches the nodes that attend it alone.  The drafts' K and V are not in the
 * cache (a rejected draft leaves no trace in the pages or their scales); store what
 * is accepted with dora_kv_append_path.
 *   desc         as for dora_decode_attn; seq_lens counts the cached tokens only;
 *                num_waves (0 = library default) is rounded up to workgroups of 2 or 4,
 *                min_range_pages is not used
 *   num_nodes    T in [1, 64]
 *   q, out       device bf16 [B][T][Hq][d]
 *   k_draft, v_draft  device bf16 [B][T][Hkv][d], 16-byte aligned
 *   tree_mask    device uint64 [B][T]
 *   node_counts  device int32 [B] in [0, T], or NULL (all T; values outside are
 *                taken as the nearest inside)
 *   workspace    >= dora_decode_tree_workspace_bytes(desc, num_nodes) bytes
 * Other arguments, flags and errors as for dora_decode_attn.  Repeated calls on the
 * same inputs and device are bitwise identical. */
size_t dora_decode_tree_workspace_bytes(const dora_decode_desc* desc, int32_t num_nodes);
dora_status dora_decode_attn_tree(const dora_decode_desc* desc, int32_t num_nodes, const void* q,
                                  const void* k_draft, const void* v_draft,
                                  const uint64_t* tree_mask, const int32_t* node_counts,
                                  const void* k_pages, const void* v_pages,
                                  const int32_t* block_table, const int32_t* seq_lens,
                                  const int32_t* version_ids, void* out, void* workspace,
                                  size_t workspace_bytes, dora_stream_t stream);

/* Decode attention with a sliding window and sinks: the operation of
 * dora_decode_attn over the tokens t < L of sequence b with
 *   t < sinks  or  t >= L - window
 * alone.  Only the pages that hold such tokens are read, and only their table entries:
 * the others may hold anything (dora_pool_release_window frees their pages).
 *   window       >= 1 (the newest token counts among them)
 *   sinks        >= 0
 *   desc         as for dora_decode_attn; num_waves and min_range_pages are not used;
 *                DORA_FLAG_VALIDATE checks the entries that are read
 *   workspace    >= dora_decode_window_workspace_bytes(desc, window, sinks) bytes
 * Other arguments, flags and errors as for dora_decode_attn. */
size_t dora_decode_window_workspace_bytes(const dora_decode_desc* desc, int32_t window,
                                          int32_t sinks);
dora_status dora_decode_attn_window(const dora_decode_desc* desc, int32_t window, int32_t sinks,
                                    const void* q, const void* k_pages, const void* v_pages,
                                    const int32_t* block_table, const int32_t* seq_lens,
                                    const int32_t* version_ids, void* out, void* workspace,
                                    size_t workspace_bytes, dora_stream_t stream);

/* Store every sequence's current-token K and V into its page slot: the write
 * that precedes each decode step (the per-token step of Sec. 2.2; seq_lens
 * counts that token, so dora_decode_attn with the same seq_lens then attends
 * over it).  Token t = seq_lens[b] - 1 of sequence b goes to page
 * block_table[b][t / P], token slot t % P; seq_lens[b] = 0 appends nothing.
 *   desc         the decode descriptor (num_seqs, num_kv_heads, head_dim,
 *                page_size, block_table_stride, num_pages, kv_dtype; flags may
 *                hold DORA_FLAG_VALIDATE; num_q_heads must be valid for it)
 *   k_new, v_new device bf16 [B][Hkv][d], 16-byte aligned
 *   block_table, seq_lens, version_ids  as for dora_decode_attn
 *   k_pages, v_pages  device, the layouts above, written in place
 *   k_scales, v_scales  device fp32 [num_pages], fp8 only (else ignored),
 *                updated in place
 *   dev_status   device int32 or NULL: receives DORA_OK, or
 *                DORA_ERR_DEVICE_CHECK if some sequence was skipped because its
 *                page id is out of range, its length exceeds its block-table
 *                row, or (under DORA_FLAG_VALIDATE with desc->page_owner) its
 *                page belongs to another version.  Skipped sequences write
 *                nothing; no write ever leaves the pool.
 * bf16 pages take the values as given.  fp8 pages: the paper fixes no
 * quantisation policy; this library keeps one fp32 scale per page for K and one
 * for V, grow-only, computed in fp32 with IEEE rounding:
 *   amax = max |x| over the token's Hkv x d values
 *   fresh = max(amax / 448, 2^-126)   (a normal fp32 number)
 *   slot 0:                           s = fresh
 *   slot > 0, not fresh <= s0:        s = fresh, and every earlier code c of
 *                                     the page (all heads) becomes
 *                                     enc((dec(c) * s0) / s)
 *   otherwise:                        s = s0       (s0: the page's scale)
 *   codes of the token: enc(x / s); the page's scale becomes s.
 * enc is the nearest OCP E4M3FN code, ties to even, saturating at +-448.
 * 4-bit pages: no token depends on another.  With top the largest magnitude,
 *   K, for each 32 dims: e = clamp(((bits of bf16 top + 0x20) >> 7) - 2, 1, 252) is the
 *      exponent stored (top's own, less 2, and one more where its mantissa is 1.75 or
 *      above), the codes are enc4(x / 2^(e - 127))
 *   V, for each 64 dims: s = max(bf16(fp32(top / 6)), 2^-126), the codes are
 *      enc4(fp32(x / s)); an infinite top counts as bf16's largest number
 * enc4 is the nearest E2M1 value, ties to the even code, +-6 beyond (infinities too).
 * A NaN makes its block NaN (exponent 255 or a NaN scale, codes 0).  The other half
 * of a byte that holds two tokens' codes stays as it is.
 * The pages of one call must belong to distinct sequences (a page is never
 * appended to by two sequences at once).  Enqueued on `stream`; one launch
 * (two with dev_status). */
dora_status dora_kv_append(const dora_decode_desc* desc, const void* k_new, const void* v_new,
                           const int32_t* block_table, const int32_t* seq_lens,
                           const int32_t* version_ids, void* k_pages, void* v_pages,
                           float* k_scales, float* v_scales, int32_t* dev_status,
                           dora_stream_t stream);

/* Store several tokens of every sequence: the accepted path of a tree of drafts, or a
 * run of a prompt.  With n = counts[b] (num_tokens without counts) and L =
 * seq_lens[b], which counts them, token i < n is row path[b][i] (row i without path) of
 * k_new[b] and v_new[b] and goes to position L - n + i.  The pages and scales end up as
 * after n calls of dora_kv_append, one token each in that order, bit for bit (only the sign
 * of a NaN code of a page whose scale is NaN is open).  As there, the pages of one call must
 * belong to distinct sequences; a page's other slots may be read and written back.
 *   num_tokens   T in [1, DORA_PATH_MAX_TOKENS], rows of k_new and v_new per sequence
 *   k_new, v_new device bf16 [B][T][Hkv][d], 16-byte aligned
 *   path         device int32 [B][T] or NULL; entries i >= n are not read; an index
 *                may occur more than once
 *   counts       device int32 [B] in [0, T] or NULL
 *   dev_status   device int32 or NULL: receives DORA_OK, or DORA_ERR_DEVICE_CHECK if
 *                something was skipped: a sequence whose n is negative or above T or L,
 *                or whose length exceeds its block-table row; a page whose id is out of
 *                range (or, under DORA_FLAG_VALIDATE with desc->page_owner, another
 *                version's); a page with a token whose path entry is no row.  A skipped
 *                sequence or page is left as it was; no write ever leaves the pool.
 * Other arguments as for dora_kv_append.  Enqueued on `stream`; one launch (two with
 * dev_status). */
#define DORA_PATH_MAX_TOKENS (1 << 19)
dora_status dora_kv_append_path(const dora_decode_desc* desc, int32_t num_tokens,
                                const void* k_new, const void* v_new, const int32_t* path,
                                const int32_t* counts, const int32_t* block_table,
                                const int32_t* seq_lens, const int32_t* version_ids, void* k_pages,
                                void* v_pages, float* k_scales, float* v_scales,
                                int32_t* dev_status, dora_stream_t stream);

/* Read the last tokens of every sequence back as bf16 rows: for n = counts[b]
 * (num_tokens without counts) and L = seq_lens[b], row i < n of k_out[b] and v_out[b] is
 * token L - n + i; rows behind it are left as they were.  bf16 pages give the values as
 * they are; fp8 (code * scale) and 4-bit V (code * scale) are fp32 products rounded to
 * bf16, 4-bit K is exact.
 *   num_tokens   T in [1, DORA_PATH_MAX_TOKENS], rows of k_out and v_out per sequence
 *   k_out, v_out device bf16 [B][T][Hkv][d], 16-byte aligned
 *   counts       device int32 [B] in [0, T], or NULL
 *   dev_status   as for dora_kv_append_path: what is skipped writes nothing
 * The fp8 scales are desc's. */
dora_status dora_kv_read(const dora_decode_desc* desc, int32_t num_tokens, const int32_t* counts,
                         const void* k_pages, const void* v_pages, const int32_t* block_table,
                         const int32_t* seq_lens, const int32_t* version_ids, void* k_out,
                         void* v_out, int32_t* dev_status, dora_stream_t stream);

/* ---------------------------------------------------------------------------
 * Attention over the pages that a query wants most.  For a long sequence a step
 * reads the bounds of its pages instead of the pages, chooses the pages that
 * the bounds promise the largest scores, for each KV head, and attends those:
 *   dora_kv_append[_path], then dora_kv_page_bounds over the same tokens;
 *   dora_page_select; dora_decode_attn_pages.
 * ------------------------------------------------------------------------- */

/* Bytes of one page's bounds: for each KV head int8 [2][d], the largest and the smallest value
 * of each dim in units of a scale, then, behind those of all heads, an fp32 scale for each;
 * rounded up to 16.  0 for an unsupported geometry. */
size_t dora_page_bounds_bytes(int32_t num_kv_heads, int32_t head_dim);

/* Bounds of the keys of every page that the last n = counts[b] (num_tokens without counts)
 * tokens of a sequence lie in, over the page's tokens t < L = seq_lens[b] (those before the
 * last n too).  For each KV head, in fp32 with IEEE rounding, over the page's keys x:
 *   s = max(max |x| / 127, 2^-126), largest[d] = ceil(max x_d / s), smallest[d] =
 *   floor(min x_d / s), within +-127
 * where a NaN (of 4-bit pages, a NaN block) counts as 0 and an infinity as bf16's largest
 * number.  The calls that move pages (dora_kv_page_copy, pack, unpack) leave bounds to the
 * caller: records of pages that dora_pool_compact or a migration moves whole are copied with
 * them, or taken again; a fork's own page, which may hold fewer tokens than the page it was
 * copied from, has its bounds taken again; those of a page that is given to another
 * sequence are taken as its tokens are appended.
 *   num_tokens   in [1, DORA_PATH_MAX_TOKENS]
 *   bounds       device [num_pages] records of dora_page_bounds_bytes, 16-byte aligned
 *   dev_status   as for dora_kv_append_path; a page that is skipped keeps its bounds
 * The fp8 scales are desc's (v_scales is not used). */
dora_status dora_kv_page_bounds(const dora_decode_desc* desc, int32_t num_tokens,
                                const int32_t* counts, const void* k_pages,
                                const int32_t* block_table, const int32_t* seq_lens,
                                const int32_t* version_ids, void* bounds, int32_t* dev_status,
                                dora_stream_t stream);

/* Choose the pages that each (sequence, KV head) reads.  With N the pages of a sequence:
 * all of them where N <= budget; else the first sink_pages, the last recent_pages, and of
 * those between the budget - sink_pages - recent_pages with the largest scores (of equal
 * ones the lower page).  The score of page j for KV head g is
 *   s * max over the group's rows h of fp32(r_h * sum_d max(u_hd lo_d, u_hd hi_d))
 * with hi, lo, s the page's bounds and the row as whole numbers u_hd = rint(q_hd / r_h), r_h
 * = max(max |q_h| / 127, 2^-126): each operation in fp32 with IEEE rounding, the sum exact.
 * So the choice depends on nothing but its inputs.  A NaN of q counts as 0, an infinity as
 * bf16's largest number.
 *   desc         num_seqs, heads, head_dim, page_size, block_table_stride, num_pages;
 *                kv_dtype and scales are not used; DORA_FLAG_VALIDATE checks the tables
 *   budget       pages of a list, >= max(1, sink_pages + recent_pages), < 2^19
 *   q            device bf16 [B][Hq][d]
 *   bounds       device, as dora_kv_page_bounds writes them
 *   page_lists   device int32 [B][Hkv][budget]: numbers of the sequence's pages (places in its
 *                table's row), ascending; entries behind the count are left as they were
 *   page_counts  device int32 [B][Hkv]: min(N, budget)
 *   scores       device fp32 [B][Hkv][block_table_stride] or NULL: receives the scores of the
 *                sequence's pages (entries behind them are left as they were)
 *   workspace    >= dora_page_select_workspace_bytes(desc) bytes (with scores, 256), 16-byte aligned
 * One launch where rows are few and short, else two. */
size_t dora_page_select_workspace_bytes(const dora_decode_desc* desc);
dora_status dora_page_select(const dora_decode_desc* desc, int32_t budget, int32_t sink_pages,
                             int32_t recent_pages, const void* q, const void* bounds,
                             const int32_t* block_table, const int32_t* seq_lens,
                             const int32_t* version_ids, int32_t* page_lists,
                             int32_t* page_counts, float* scores, void* workspace,
                             size_t workspace_bytes, dora_stream_t stream);

/* Decode attention over listed pages: the operation of dora_decode_attn over the tokens t <
 * seq_lens[b] of the pages page_lists[b][g][i], i < page_counts[b][g], alone, g the KV head.
 * A list may be in any order; a page listed twice counts twice; an entry that is no page of
 * the sequence (negative, or at or behind its last token) counts for nothing.  A row that
 * attends nothing gives 0.  Only the table entries of listed pages are read.
 *   list_stride  entries of a list, in [1, 2^19)
 *   page_lists   device int32 [B][Hkv][list_stride], numbers of the sequence's pages
 *   page_counts  device int32 [B][Hkv] in [0, list_stride] (values outside are taken as the
 *                nearest inside)
 *   desc         as for dora_decode_attn, any kv_dtype; num_waves and min_range_pages are not
 *                used; DORA_FLAG_VALIDATE checks counts, entries and the listed pages' ids
 *   workspace    >= dora_decode_pages_workspace_bytes(desc, list_stride) bytes
 * Other arguments, flags and errors as for dora_decode_attn.  Repeated calls on the same inputs
 * are bitwise identical. */
size_t dora_decode_pages_workspace_bytes(const dora_decode_desc* desc, int32_t list_stride);
dora_status dora_decode_attn_pages(const dora_decode_desc* desc, int32_t list_stride,
                                   const void* q, const int32_t* page_lists,
                                   const int32_t* page_counts, const void* k_pages,
                                   const void* v_pages, const int32_t* block_table,
                                   const int32_t* seq_lens, const int32_t* version_ids, void* out,
                                   void* workspace, size_t workspace_bytes, dora_stream_t stream);

/* ---------------------------------------------------------------------------
 * KV page pack / unpack: the device half of the paper's two-phase state
 * transfer for same-version migration (Sec. 3.4: request metadata travels by
 * RPC, the KV data by collectives; KV states are equal on every instance of
 * the version, so no re-prefill).
 *
 * Packed buffer format (all integers little-endian):
 *   bytes [0, 256)   header:
 *       0  char[8]  magic "DORAKV01"
 *       8  int32    format (= 1)
 *      12  int32    policy_version
 *      16  int32    kv_dtype
 *      20  int32    page_size
 *      24  int32    num_kv_heads
 *      28  int32    head_dim
 *      32  int64    n_pages
 *      40  int64    page_bytes   (= num_kv_heads * page_size * head_dim * e; of
 *                                 4-bit pages e = 17 / 32)
 *      48  int32    n_seqs       (caller's count of sequences in the list)
 *      52  int32    reserved (0); bytes 56..255 are 0
 *   then n_pages K pages (page_bytes each) in list order,
 *   then n_pages V pages in list order,
 *   then, for fp8 only, n_pages fp32 k scales and n_pages fp32 v scales.
 * Pages are copied whole, tail slots included; the copy is bit-exact.
 * ------------------------------------------------------------------------- */

typedef struct {
  int32_t kv_dtype;        /* dora_kv_dtype */
  int32_t page_size;
  int32_t num_kv_heads;
  int32_t head_dim;
  int64_t num_pages;       /* capacity of the pool the page ids index */
  int32_t policy_version;  /* version tag of the pages (pack: source, unpack: destination) */
  int32_t n_seqs;          /* recorded in the header by pack; informational */
} dora_pack_desc;

/* Size in bytes of a packed buffer holding n_pages pages (0 if invalid). */
size_t dora_kv_packed_bytes(const dora_pack_desc* desc, int64_t n_pages);

/* Gather pages src_pages[0..n_pages) (device int32, logical order) of a pool
 * into `packed` (>= dora_kv_packed_bytes bytes, 16-byte aligned) and write the
 * header.  k_scales/v_scales: device [num_pages], fp8 only.
 * `packed` may be device memory, or pinned host memory from hipHostMalloc
 * (mapped: the kernel writes it over the host link).  The latter is the
 * offload half of the paper's hierarchical memory management (Sec. 3.4: KV
 * caches moved to host memory under VRAM pressure and restored for deferred
 * generation); no device staging buffer is needed. */
dora_status dora_kv_page_pack(const dora_pack_desc* desc,
                              const void* k_pages, const void* v_pages,
                              const float* k_scales, const float* v_scales,
                              const int32_t* src_pages, int64_t n_pages,
                              void* packed, size_t packed_bytes,
                              dora_stream_t stream);

/* Scatter a packed buffer into pages dst_pages[0..n_pages) (device int32) of
 * the destination pool described by `desc`.  src_version is the version tag the
 * request metadata carries; it must equal desc->policy_version, else
 * DORA_ERR_VERSION_MISMATCH before any launch (KV states are only equivalent
 * within one policy version).  On the device the header is checked against
 * desc and n_pages; on any mismatch nothing is written to the pool and, if
 * dev_status (device int32, may be NULL) is given, it receives a non-zero
 * dora_status code; it receives DORA_OK otherwise.  `packed` may be device
 * memory or pinned host memory from hipHostMalloc (restore from host: the
 * kernel reads it over the host link). */
dora_status dora_kv_page_unpack(const dora_pack_desc* desc, int32_t src_version,
                                const void* packed, size_t packed_bytes,
                                const int32_t* dst_pages, int64_t n_pages,
                                void* k_pages, void* v_pages,
                                float* k_scales, float* v_scales,
                                int32_t* dev_status, dora_stream_t stream);

/* Copy pages inside one pool: page dst_pages[i] becomes a copy of page src_pages[i]
 * (K, V and, for fp8, its scales), bit for bit, for i < n_pages (device int32 lists).
 * The device half of dora_pool_fork_seq and dora_pool_compact, which make the lists.
 * A page may be copied to many places, and onto itself (nothing happens); the
 * destinations must differ from each other, and none may be the source of another
 * copy.  desc->policy_version and n_seqs are not used.  dev_status (device int32 or
 * NULL) receives DORA_OK, or DORA_ERR_DEVICE_CHECK if a pair was skipped because one
 * of its ids is out of range. */
dora_status dora_kv_page_copy(const dora_pack_desc* desc, void* k_pages, void* v_pages,
                              float* k_scales, float* v_scales, const int32_t* src_pages,
                              const int32_t* dst_pages, int64_t n_pages, int32_t* dev_status,
                              dora_stream_t stream);

/* ---------------------------------------------------------------------------
 * Orchestrator planners (host, integer arithmetic; Sec. 3.3).  Versions are
 * indexed oldest first; the last index is the latest version.
 * ------------------------------------------------------------------------- */

/* Resource partitioning plan: DP groups per version in proportion to its
 * workload (active plus pending requests).  A version with work keeps at least
 * one group; the other groups go by the largest-remainder method on the
 * quotas (n_groups - busy versions) * workload / total, equal remainders to the
 * newer version; with no work, every group goes to the latest version.
 *   workload    host int64 [n_versions], >= 0
 *   groups_out  host int32 [n_versions], sums to n_groups
 * DORA_ERR_INVALID_ARG for null pointers, negative workload, n_groups < 1, or
 * more versions with work than groups. */
dora_status dora_plan_partition(const int64_t* workload, int32_t n_versions, int32_t n_groups,
                                int32_t* groups_out);

/* Staleness-aware data supplementation: prompts to inject per version.  The
 * latest version gets min(latest_quota, its idle slots), latest_quota being
 * what its rollout batch still needs; every legacy version gets exactly its
 * residual idle slots (groups * slots_per_group - active, at least 0).
 *   groups, active  host int32 [n_versions], >= 0
 *   inject_out      host int32 [n_versions] */
dora_status dora_plan_supplement(const int32_t* groups, const int32_t* active,
                                 int32_t n_versions, int32_t slots_per_group,
                                 int64_t latest_quota, int32_t* inject_out);

/* ---------------------------------------------------------------------------
 * Host page pool: page allocator plus per-version sequence tables for one
 * shared pool (Sec. 3.2: every request carries its version tag; Sec. 3.3: the
 * orchestrator reads per-version KV-cache utilisation; Sec. 3.4: migration
 * only between instances of the same version, locality first).  Metadata only:
 * the pool never touches device memory.  Not thread-safe.
 * ------------------------------------------------------------------------- */

typedef struct dora_pool dora_pool;

/* num_pages >= 1, page_size >= 1, num_versions >= 1.  seed != 0 shuffles the
 * free list with a seeded generator so that pages are scattered in the pool;
 * seed == 0 hands pages out in increasing order. */
dora_status dora_pool_create(int64_t num_pages, int32_t page_size,
                             int32_t num_versions, uint64_t seed, dora_pool** out);
void        dora_pool_destroy(dora_pool* pool);

/* Register a sequence of `version` holding num_tokens tokens and allocate its
 * ceil(num_tokens / page_size) pages.  DORA_ERR_POOL_EXHAUSTED leaves the pool
 * unchanged. */
dora_status dora_pool_add_seq(dora_pool* pool, int32_t version, int32_t num_tokens,
                              int64_t* seq_id_out);
/* Grow a sequence to new_num_tokens (>= current), allocating pages as needed. */
dora_status dora_pool_extend_seq(dora_pool* pool, int64_t seq_id, int32_t new_num_tokens);
/* Release a sequence; its pages are free once no other sequence holds them. */
dora_status dora_pool_free_seq(dora_pool* pool, int64_t seq_id);
/* Tokens, version and page count of a sequence (any out pointer may be NULL). */
dora_status dora_pool_seq_info(const dora_pool* pool, int64_t seq_id, int32_t* num_tokens,
                               int32_t* version, int32_t* num_pages);
/* Copy a sequence's page ids in logical order into pages_out[cap]; -1 stands for a
 * page that dora_pool_release_window has released. */
dora_status dora_pool_seq_pages(const dora_pool* pool, int64_t seq_id,
                                int32_t* pages_out, int32_t cap, int32_t* n_out);
/* Fill host arrays for a decode batch: table_out[n][stride] (entries that are unused,
 * or whose page is released, set to 0), lens_out[n], versions_out[n].  INVALID_ARG if a sequence needs
 * more than `stride` pages. */
dora_status dora_pool_block_table(const dora_pool* pool, const int64_t* seq_ids, int32_t n,
                                  int32_t stride, int32_t* table_out, int32_t* lens_out,
                                  int32_t* versions_out);
/* owner_out[num_pages]: owning version of each page, -1 if free. */
dora_status dora_pool_page_owner(const dora_pool* pool, int16_t* owner_out);
/* Pages held by `version` (version = -1: all versions; a page that several sequences
 * share counts once) and pages free. */
dora_status dora_pool_stats(const dora_pool* pool, int32_t version, int64_t* pages_used,
                            int64_t* pages_free);
/* Migrate a sequence from `src` to `dst` (same-version instances): allocates
 * pages in dst for dst_version and registers the sequence there; writes the
 * source page list and the destination page list (logical order, n_out
 * entries each) for pack/unpack, and the new id.  dst_version must equal the
 * sequence's version (DORA_ERR_VERSION_MISMATCH otherwise).  If src == dst the
 * sequence stays where it is (locality: no pages move, n_out = 0 and
 * dst_seq_id = seq_id).  The source sequence is kept until the caller frees it
 * after the copy.  Pages shared with other sequences are copied for the migrated one;
 * released pages stay released. */
dora_status dora_pool_migrate_seq(dora_pool* src, int64_t seq_id, dora_pool* dst,
                                  int32_t dst_version, int64_t* dst_seq_id,
                                  int32_t* src_pages, int32_t* dst_pages, int32_t cap,
                                  int32_t* n_out);

/* Fork a sequence: register a new one, of the same version, that holds the first
 * num_tokens tokens (0 <= num_tokens <= the sequence's; all of them where the sequence
 * has released pages, else DORA_ERR_INVALID_ARG).  It shares the pages that these
 * fill, and gets a page of its own for the last, partly filled one: then *n_out = 1 and
 * the page must be copied from *src_page to *dst_page with dora_kv_page_copy before
 * either sequence is appended to (n_out = 0: nothing to copy; released pages stay
 * released).  Shared pages are what dora_decode_attn_grouped reads once.
 * DORA_ERR_POOL_EXHAUSTED leaves the pool unchanged. */
dora_status dora_pool_fork_seq(dora_pool* pool, int64_t seq_id, int32_t num_tokens,
                               int64_t* new_seq_id, int32_t* src_page, int32_t* dst_page,
                               int32_t* n_out);
/* Release the pages of a sequence that no later dora_decode_attn_window call with this
 * window and these sinks reads (window >= 1, sinks >= 0): those that lie whole between
 * the sinks and the window of the newest token.  Its tokens still count, its table keeps
 * its width; it is for dora_decode_attn_window from then on.  Call it once the tokens that
 * the sequence counts are stored: dora_kv_append_path of more of them than the window holds
 * would find 0 for a released page, and write what may be another sequence's.
 * *n_out (may be NULL): pages released by this sequence in this call. */
dora_status dora_pool_release_window(dora_pool* pool, int64_t seq_id, int32_t window,
                                     int32_t sinks, int32_t* n_out);
/* Move live pages from the pool's end into its free places, so that the n live pages
 * are pages 0 .. n - 1: fills src_pages and dst_pages (cap entries; *n_out of them) for
 * one dora_kv_page_copy per layer and renames the pages in every sequence; block tables
 * taken before are stale, and so are page ids of forks and migrations whose copies are not
 * yet made.  Afterwards pages are handed out in increasing order.
 * DORA_ERR_WORKSPACE_TOO_SMALL (more than cap moves; *n_out says how many) leaves the
 * pool unchanged. */
dora_status dora_pool_compact(dora_pool* pool, int32_t* src_pages, int32_t* dst_pages, int32_t cap,
                              int32_t* n_out);

#ifdef __cplusplus
}
#endif

#endif /* DORA_H */
