// Entry point of attention over a paged cache: checks, and which kernel runs.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "attn_general.h"
#include "attn_launch.h"

namespace {

using namespace bitcos_attn;

// Workers that share a launch's key tiles on 256 CUs: eight waves a CU for few
// query rows (1024 / 1536 / 2048 / 2560 workers: 64 ragged requests 149 / 140 /
// 139 / 149 us, 32 long ones 383 / 328 / 297 / 320 us), two workgroups of four
// waves for many (256 / 512 / 1024: a prompt of 8192 898 / 642 / 650 us, a chunk
// beside 16 single tokens 64 / 58 / 67 us), three where a head has 64 values,
// whose rows and tiles take half the registers and LDS (a prompt of 8192, 24/4
// heads, two / three: bfloat16 363 / 329 us, int8 420 / 399 us).
constexpr int kWaves = 2048, kGroups = 512, kGroups64 = 768;

int launch_general(const AttnArgs& A, hipStream_t stream) {
  const int64_t rows = static_cast<int64_t>(A.tokens) * A.q_heads;
  const int64_t blocks = std::min<int64_t>((rows + 3) / 4, 1 << 20);
  const auto fn = A.c.dtype == BITCOS_KV_I8 ? paged_attn_general_kernel<int8_t> : paged_attn_general_kernel<__bf16>;
  hipLaunchKernelGGL(fn, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, A);
  return bitcos_launch_status();
}

// The shapes the matrix-core kernels take, as far as the counts tell.
AttnPlan plan_of(const bitcos_kv_cache* c, int32_t tokens, int32_t requests, int32_t q_heads, int32_t max_q, int32_t max_kv) {
  AttnPlan p{};
  p.bytes = 16;
  const int group = q_heads / c->kv_heads, elem = c->dtype == BITCOS_KV_I8 ? 1 : 2;
  if (q_heads % c->kv_heads || (c->head_dim != 64 && c->head_dim != 128)) return p;
  if (c->page_size < 16 || (c->page_size & (c->page_size - 1))) return p;
  if (!rows_aligned16(c->k, c->k_stride, 3, elem) || !rows_aligned16(c->v, c->v_stride, 3, elem)) return p;
  // Within a page, and from page to page, 32 bits of bytes.
  for (const int64_t* st : {c->k_stride, c->v_stride})
    if (st[2] > (1 << 24) || st[2] * c->page_size * elem > INT32_MAX || st[0] * elem > UINT32_MAX) return p;
  if (4ll * c->kv_heads * c->page_size > UINT32_MAX) return p;
  if (group > 128) return p;
  const int64_t want = static_cast<int64_t>(std::min(max_q, tokens)) * group;
  // Rows that a wave's registers hold.  Drafted tokens, 24 requests of 30 to 6000 keys / 64 of 30 to 16000, here and in the
  // other kernel, us: 128 values, 30 rows, bfloat16 70 / 320 and 67 / 336, int8 56 / 211 and 58 / 264; 5 rows 54 / 286 and
  // 58 / 323, int8 39 / 166 and 55 / 263; 40 rows, which would spill here, 127 / 506 and 69 / 345.  64 values, 30 rows,
  // bfloat16 31 / 92 and 26 / 97, int8 32 / 79 and 29 / 83; 48 rows 39 / 104 and 29 / 103, int8 42 / 112 and 31 / 96: those
  // stay here for their weights' digits, not for speed.
  // (Single tokens beside a chunk go to the other kernel with it: launches of their own took 70 us where the mixture takes 57.)
  const int few = c->head_dim == 64 ? 64 : 32;
  p.tiles = want > few || group > few ? 0 : want <= 16 ? 1 : want <= 32 ? 2 : 4;
  p.tt = std::min((p.tiles ? 16 * p.tiles : 128) / group, max_q);
  p.rows = static_cast<int64_t>(p.tt) * group;
  p.page_shift = __builtin_ctz(c->page_size);
  // A part costs what its rows' sums cost to write and read again, a tile of a worker's own some 2 us: with up to 16 rows
  // one tile each is best for short lists (2000 keys: 12.5 us, two each 13.7), with more rows four (24 requests of 5
  // tokens: 22.7 us; two each 23.2, eight 32.4).
  p.least_log2 = p.tiles == 1 ? 0 : 2;
  const int64_t items = (static_cast<int64_t>(tokens) / p.tt + requests) * c->kv_heads;
  const int64_t units = items * (max_kv / (p.tiles ? 32 : 64) + 2);
  p.most = static_cast<int>(std::min<int64_t>(p.tiles ? kWaves : c->head_dim == 64 ? kGroups64 : kGroups, (units >> p.least_log2) + 1));
  p.matrix = true;
  p.bytes = 16 * static_cast<size_t>(p.most) + static_cast<size_t>(p.most) * 2 * p.rows * (c->head_dim + 2) * 4;
  return p;
}

}  // namespace

extern "C" size_t bitcos_paged_attn_workspace(const bitcos_kv_cache* cache, int32_t tokens, int32_t requests,
                                              int32_t q_heads, int32_t max_q, int32_t max_kv) {
  if (kv_cache_status(cache) || tokens < 1 || requests < 1 || q_heads < 1 || max_q < 1 || max_kv < 0) return 0;
  return plan_of(cache, tokens, requests, q_heads, max_q, max_kv).bytes;
}

extern "C" int bitcos_paged_attn(const bitcos_kv_cache* cache, int32_t tokens, int32_t requests, int32_t q_heads,
                                 const void* q, const int64_t* q_stride, const int32_t* table, int32_t table_width,
                                 const int32_t* kv_len, const int32_t* cu_q, int32_t max_q, int32_t max_kv, float scale,
                                 int32_t causal, int32_t window, void* out, const int64_t* out_stride, float* lse,
                                 void* ws_dev, size_t ws_bytes, void* stream) {
  if (const int st = kv_cache_status(cache)) return st;
  if (!q || !q_stride || !table || !kv_len || !cu_q || !out || !out_stride || !ws_dev) return BITCOS_E_ARG;
  if (tokens < 1 || requests < 1 || requests == INT32_MAX || q_heads < 1 || q_heads % cache->kv_heads) return BITCOS_E_ARG;
  if (table_width < 1 || static_cast<int64_t>(table_width) * cache->page_size > INT32_MAX) return BITCOS_E_ARG;
  if (max_q < 1 || max_kv < 0 || window < 0 || !std::isfinite(scale)) return BITCOS_E_ARG;
  for (int i = 0; i < 2; ++i)
    if (q_stride[i] < 0 || out_stride[i] < 0) return BITCOS_E_ARG;
  if (reinterpret_cast<uintptr_t>(ws_dev) % 16) return BITCOS_E_ARG;
  const AttnPlan p = plan_of(cache, tokens, requests, q_heads, max_q, max_kv);
  if (ws_bytes < p.bytes) return BITCOS_E_SPACE;
  AttnArgs A{};
  A.c = *cache;
  A.q = static_cast<const uint16_t*>(q);
  A.table = table;
  A.kv_len = kv_len;
  A.cu_q = cu_q;
  A.out = static_cast<uint16_t*>(out);
  A.lse = lse;
  for (int i = 0; i < 2; ++i) A.qs[i] = q_stride[i], A.os[i] = out_stride[i];
  A.tokens = tokens;
  A.requests = requests;
  A.q_heads = q_heads;
  A.group = q_heads / cache->kv_heads;
  A.width = table_width;
  A.kv_max = table_width * cache->page_size;
  A.window = window;
  A.causal = causal != 0;
  A.scale = scale;
  // The schedule divides units (at most these) in doubles.
  const bool countable = (static_cast<double>(tokens) + requests) * cache->kv_heads * (A.kv_max / 32.0 + 2) < 1099511627776.0;
  // The matrix-core kernels form the numbers of up to 64 tiles of keys past the last in 32 bits.
  const bool numbered = A.kv_max <= INT32_MAX - 8192;
  if (p.matrix && countable && numbered && rows_aligned16(q, q_stride, 2, 2) && rows_aligned16(out, out_stride, 2, 2)) {
    A.tt = p.tt;
    A.tt_inv = ~uint64_t{0} / static_cast<uint64_t>(p.tt) + 1;
    A.group_inv = (65536 + A.group - 1) / A.group;
    A.page_shift = p.page_shift;
    Parts P;
    P.note = static_cast<int4*>(ws_dev);
    P.rows = static_cast<int32_t>(p.rows);
    P.acc = reinterpret_cast<float*>(P.note + p.most);
    P.ml = P.acc + 2ll * p.most * p.rows * cache->head_dim;
    return (p.tiles ? attn_decode_launch : attn_chunk_launch)(A, p, P, static_cast<hipStream_t>(stream));
  }
  return launch_general(A, static_cast<hipStream_t>(stream));
}
