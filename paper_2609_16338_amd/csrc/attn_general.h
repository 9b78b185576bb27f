// Attention for any head size, page size, stride and alignment: one wave per
// (query, head), all its keys (attn_rows.h).  Bound by the latency of reads
// that do not coalesce; it stands for shapes that are rare, not for speed (one
// request of 2000 keys, 32/8 heads: of 128 values 19 us by the matrix cores, of
// 96 975 here, of 256 1940; a prompt of 1000 52, 3170, 7870 us).
#pragma once

#include "attn_rows.h"

namespace bitcos_attn {

// T: __bf16 or int8_t.
template <class T>
__global__ void __launch_bounds__(256) paged_attn_general_kernel(AttnArgs A) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = static_cast<int64_t>(A.tokens) * A.q_heads;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + wave; row < rows; row += static_cast<int64_t>(gridDim.x) * 4) {
    const int t = static_cast<int>(row / A.q_heads), head = static_cast<int>(row - static_cast<int64_t>(t) * A.q_heads);
    // The last request that starts at or before the token (bisection; cu_q ascends).
    int a = 0, b = A.requests;
    while (b - a > 1) {
      const int mid = (a + b) >> 1;
      if (A.cu_q[mid] <= t)
        a = mid;
      else
        b = mid;
    }
    const Span S = span_of(A, a);
    if (t < S.q0 || t >= S.q0 + S.n) continue;
    int lo, hi;
    seen(A, S, t - S.q0, lo, hi);
    row_out(A, row_over_keys<T>(A, a, t, head, head / A.group, lo, hi), t, head);
  }
}

}  // namespace bitcos_attn
