/*
 * bitcos_kv.h -- C ABI of libbitcos: the paged key/value cache of a decode engine.
 *
 * Between the q/k/v projections and the output projection of a decoder layer
 * (both GEMVs of bitcos.h) stand three steps, on sequences whose keys and
 * values lie in pages of a shared pool:
 *   bitcos_kv_plan     once per step: pages for the new tokens, the slot and
 *                      position of each, the pages of finished requests back;
 *   bitcos_kv_append   per layer: rotate and round the new q and k, store k
 *                      and v in the cache (bf16, or int8 with a scale per row);
 *   bitcos_paged_attn  per layer: softmax attention of the new tokens over the
 *                      cached ones.
 *
 * The conventions of bitcos.h hold: status codes, no aborts, validation before
 * anything is enqueued, the caller owns every buffer and the stream, nothing
 * is allocated on the device, no call synchronises.  Lengths, tables and slots
 * are device data that the host does not see: the kernels check every index
 * that they form from them against the sizes given here, so values out of
 * range lead to skipped work, as stated at each call, and never to an access
 * outside the buffers.
 */
#ifndef BITCOS_KV_H
#define BITCOS_KV_H

#include <stddef.h>
#include <stdint.h>

#include "bitcos.h"

#ifdef __cplusplus
extern "C" {
#endif

#define BITCOS_KV_BF16 1 /* keys and values bfloat16                                     */
#define BITCOS_KV_I8 2   /* int8, one fp32 scale per (token, head): a value is q * scale */

#define BITCOS_ACT_F32 1  /* new q, k, v in float32 (the GEMVs' outputs) */
#define BITCOS_ACT_BF16 2 /* ... in bfloat16                             */

#define BITCOS_KV_MAX_DIM 256 /* most values per head; a multiple of 8 */

/* A paged cache of one layer.  Token `off` of page p holds, for kv head h,
 * head_dim consecutive values at k + p * k_stride[0] + h * k_stride[1] +
 * off * k_stride[2] (strides in elements), v alike; the int8 scales lie at
 * [p][h][off] of contiguous fp32 arrays [pages][kv_heads][page_size].  A slot
 * is p * page_size + off (pages * page_size < 2^31; the data may be larger
 * than 4 GB). */
typedef struct bitcos_kv_cache {
  int32_t dtype; /* BITCOS_KV_*                       */
  int32_t pages;
  int32_t kv_heads;
  int32_t page_size; /* tokens per page, any count >= 1   */
  int32_t head_dim;  /* multiple of 8, 8..256             */
  int32_t reserved;  /* 0                                 */
  int64_t k_stride[3];
  int64_t v_stride[3];
  void* k; /* device */
  void* v;
  float* k_scale; /* NULL for BITCOS_KV_BF16 */
  float* v_scale;
} bitcos_kv_cache;

/* ---- step planning ------------------------------------------------------
 * bitcos_kv_plan: from the lengths of R requests, the pages, slots and
 * positions of a step's new tokens.  Request r has kv_len[r] tokens in the
 * cache, the pages of which are the first ceil(kv_len[r] / page_size) entries
 * of row r of `table` (int32 [R][table_width]), and new_len[r] new ones;
 * new_len[r] = 0 leaves it out of the step, new_len[r] < 0 says that it is
 * finished.  Free pages wait in `ring` (int32 [ring_cap], one place for every
 * page of the pool): those at places head .. tail - 1 (mod ring_cap), in
 * order, with ring_state = {head, tail} (int64, growing).
 *   - Tokens are numbered request by request: request r's are cu_q[r] ..
 *     cu_q[r + 1] - 1 (cu_q int32 [R + 1]).
 *   - Pages that a request needs beyond its own are taken from the ring's
 *     head, request by request, and written behind its entries in table.
 *   - slots[t], positions[t] (int32 [max_tokens]): where token t goes, and its
 *     place in its sequence; -1 both for t >= cu_q[R].
 *   - kv_len_out[r] = kv_len[r] + new tokens; 0 for a finished request, whose
 *     pages go back to the ring's tail, in order (they are not taken again in
 *     the same step; its table row is left as it is).
 *   - ring_state_out = the advanced {head, tail}; counts (int32 [4]) = tokens,
 *     pages taken, pages given back, requests refused.
 * First come, first served: from the first request on whose tokens or pages
 * no longer fit (max_tokens; the pages in the ring at the start of the step),
 * none gets any; a request that would outgrow its table row is refused by
 * itself.  A refused request keeps its kv_len and has no tokens.  The pages
 * of a finished request that find no place in the ring (more free pages than
 * ring_cap) count as refused too, and kv_len_out keeps its length.
 * kv_len is read as 0 where negative and as table_width * page_size where
 * above it.  A page id outside [0, 2^31 / page_size) gives the slot -1.
 * Only places of table and ring that held nothing are written (and, of
 * kv_len_out and ring_state_out, buffers of their own): the same call again
 * gives the same results.  No buffer may overlap another.
 * Errors: E_ARG (null pointer, but slots and positions may be with
 * max_tokens = 0; count < 1, max_tokens < 0, table_width *
 * page_size >= 2^31, buffers that overlap), E_HIP. */
int bitcos_kv_plan(const int32_t* kv_len, const int32_t* new_len, int32_t requests, int32_t* table,
                   int32_t table_width, int32_t* ring, int32_t ring_cap, const int64_t* ring_state,
                   int32_t page_size, int32_t max_tokens, int32_t* cu_q, int32_t* kv_len_out,
                   int32_t* slots, int32_t* positions, int64_t* ring_state_out, int32_t* counts,
                   void* stream);

/* ---- storing new keys and values ------------------------------------------
 * bitcos_kv_append: for t < tokens, stores k[t] and v[t] ([tokens][kv_heads]
 * [head_dim], act_dtype, strides {token, head} in elements) at slots[t] of the
 * cache; with q not NULL, q_out[t] = q[t] ([tokens][q_heads][head_dim]) as
 * bfloat16, the form bitcos_paged_attn reads.
 *   - rot_dim > 0: the first rot_dim values (even) of every q and k head are
 *     rotated first, value i with value i + rot_dim / 2, by the angle whose
 *     cosine and sine stand at [positions[t]][i] of `cos` and `sin` (fp32
 *     [max_pos][rot_dim / 2], contiguous): x1 c - x2 s and x2 c + x1 s, fp32,
 *     every operation rounded by itself.  rot_dim = 0: cos, sin and positions
 *     are not read.
 *   - Rounding to bfloat16 to nearest even, or to int8 by the rule of
 *     bitcos_quantize_act over the head's values: a = max|x| / 127 (1 for a
 *     row of zeros), q = clamp(round_half_even(x / a), -127, 127), IEEE fp32
 *     divisions; the scale a goes to k_scale / v_scale.  A row with an
 *     infinite or NaN value has that scale and zeros: NaN, all of it.
 *   - A token whose slot is outside [0, pages * page_size), or (rot_dim > 0)
 *     whose position is outside [0, max_pos), is not stored; in the second
 *     case its q_out is zero.
 * Slots are distinct (the outcome for a slot named twice is one of the two
 * rows, possibly mixed); q, k, v and q_out do not overlap the cache.
 * Alignment: that of the elements.  Errors: E_ARG, E_UNSUPPORTED, E_HIP. */
int bitcos_kv_append(const bitcos_kv_cache* cache, int32_t tokens, int32_t act_dtype, const void* k,
                     const int64_t* k_stride, const void* v, const int64_t* v_stride,
                     const int32_t* slots, int32_t q_heads, const void* q, const int64_t* q_stride,
                     void* q_out, const int64_t* q_out_stride, int32_t rot_dim, const float* cos,
                     const float* sin, int32_t max_pos, const int32_t* positions, void* stream);

/* ---- attention --------------------------------------------------------------
 * bitcos_paged_attn: softmax attention of the step's tokens over the cache.
 * Request r's queries are rows cu_q[r] .. cu_q[r + 1] - 1 of q (bfloat16
 * [tokens][q_heads][head_dim], strides {token, head}); its keys and values
 * are the first kv_len[r] tokens of the pages in row r of table, the new
 * tokens' own among them (bitcos_kv_append comes first).  Query head h reads
 * kv head h / (q_heads / kv_heads).  For query i of n with kv_len keys,
 *   position p = kv_len - n + i; visible keys j: j < kv_len; causal: j <= p;
 *   window > 0: j > p - window as well;
 *   s_j = scale * sum_d q[d] k_j[d] (int8: the key's scale multiplies the sum),
 *   m = max_j s_j,  l = sum_j e^(s_j - m),
 *   out = sum_j e^(s_j - m) v_j / l   (bfloat16, strides {token, head}),
 *   lse = m + ln l                    (fp32 [tokens][q_heads], or NULL).
 * A query that sees no key gets out = 0 and lse = -infinity; one that sees
 * keys, all with the score -infinity, out = NaN (0 / 0) and lse = -infinity.
 * Keys and values that a query does not see have no part in its result,
 * whatever they hold.
 * Scores, m, l and the sums over values are fp32 (a score past 2.3e38 counts as
 * infinite); products are exact (bf16 or int8 times bf16).  The weights
 * e^(s_j - m), int8: times the value's scale, are rounded before they multiply
 * the values: to twice bfloat16's digits by a call whose min(max_q, tokens) *
 * q_heads / kv_heads is at most 32 (64 at heads of 64 values), to bfloat16 by
 * one of longer chunks (for all of its requests: a single token beside a
 * prompt as well), not at all by the general kernel.  The order of the sums is
 * fixed for a launch and its lengths, and so are the bits on a repeat.
 *   - max_q, max_kv: what the host knows of the largest n and kv_len.  They
 *     choose the kernel and its grid; the results hold for any lengths.
 *   - ws_dev: device workspace of bitcos_paged_attn_workspace bytes (for the
 *     same counts), 16-byte aligned, contents arbitrary, not shared by calls
 *     that may overlap in time.
 *   - kv_len is read as at most table_width * page_size, cu_q as at most
 *     tokens; a key in a page whose id is outside [0, pages) is not visible.
 *     Rows of out and lse that belong to no request are left as they are; where
 *     cu_q does not ascend, a row that several requests name holds a mixture of
 *     theirs or what it held.
 * Alignment: q, out and the cache 2 bytes (int8: 1); the matrix-core kernels
 * take heads of 64 and 128 values in pages of 16, 32, 64, ... tokens with up
 * to 128 query heads on a kv head, where everything lies on 16-byte boundaries
 * and a page spans less than 4 GiB (a token 2^24 elements), and tables whose
 * rows hold up to 2^31 - 8193 tokens; a general, much slower kernel takes
 * everything else (64 requests of 2000 keys, 32/8 heads: of 128 values 94 us,
 * of 96 2300, of 256 5700).  Where a sum is not finite (an infinite
 * or NaN key, value or scale within a request), its rows are done again one by
 * one, which takes many times as long.
 * Errors: E_ARG (null pointer, bad size; q_heads not a multiple of kv_heads;
 * scale not finite; window < 0), E_SPACE (ws_bytes), E_UNSUPPORTED, E_HIP. */
size_t bitcos_paged_attn_workspace(const bitcos_kv_cache* cache, int32_t tokens, int32_t requests,
                                   int32_t q_heads, int32_t max_q, int32_t max_kv);
int bitcos_paged_attn(const bitcos_kv_cache* cache, int32_t tokens, int32_t requests, int32_t q_heads,
                      const void* q, const int64_t* q_stride, const int32_t* table,
                      int32_t table_width, const int32_t* kv_len, const int32_t* cu_q, int32_t max_q,
                      int32_t max_kv, float scale, int32_t causal, int32_t window, void* out,
                      const int64_t* out_stride, float* lse, void* ws_dev, size_t ws_bytes,
                      void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BITCOS_KV_H */
