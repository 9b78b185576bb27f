// One query row over a range of keys, by one wave, for any head size, page
// size, stride and alignment.
//
// Lane l takes the score of every 64th key: the dot product with the query,
// whose values the lanes hold between them; then a running maximum and sum
// over the wave, and the sum over values with lane l owning values l, l + 64,
// ... of the head.  All in fp32 and only over keys that the query sees, so
// whatever the others hold has no part in it.  Keys are read lane by lane, not
// coalesced: it is for shapes that the matrix-core kernels do not take, and for
// what they do again where a sum is not finite.
#pragma once

#include "attn_common.h"

namespace bitcos_attn {

constexpr int kOwn = BITCOS_KV_MAX_DIM / 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The maximum of a row that sees keys, all of them with the score -infinity: its sums stay zero, and its result is 0 / 0.
// A row that sees no key has the maximum -infinity, and gives zeros.
constexpr float kLowest = -__FLT_MAX__;

// Maximum (base 2), sum of weights, and the lane's sums over values.
struct RowSums {
  float m, l, acc[kOwn];
};

// Query `head` of token t over keys [lo, hi) of request r.  T: __bf16 or int8_t.
template <class T>
__device__ __forceinline__ RowSums row_over_keys(const AttnArgs& A, int r, int64_t t, int64_t head, int kv_head, int lo, int hi) {
  constexpr bool kI8 = sizeof(T) == 1;
  const int lane = threadIdx.x & 63, dim = A.c.head_dim;
  const __bf16* q = reinterpret_cast<const __bf16*>(A.q) + t * A.qs[0] + head * A.qs[1];
  float qv[kOwn];
  RowSums R{-INFINITY, 0.0f, {}};
#pragma unroll
  for (int i = 0; i < kOwn; ++i) qv[i] = lane + 64 * i < dim ? static_cast<float>(q[lane + 64 * i]) : 0.0f;
  for (int64_t j0 = lo; j0 < hi; j0 += 64) {  // (64 keys past the last may be past 2^31)
    const int n = static_cast<int>(min(static_cast<int64_t>(64), hi - j0));
    bool on = lane < n;
    int page = -1, off = 0;
    if (on) {
      const int j = static_cast<int>(j0) + lane;
      const int p = j / A.c.page_size;
      off = j - p * A.c.page_size;
      page = A.table[static_cast<int64_t>(r) * A.width + p];
      on = page >= 0 && page < A.c.pages;
    }
    float s = -INFINITY, vs = 1.0f, dot = 0.0f;
    const T* k = static_cast<const T*>(A.c.k) + (on ? page : 0) * A.c.k_stride[0] + kv_head * A.c.k_stride[1] + off * A.c.k_stride[2];
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      for (int d = 64 * i; d < min(dim, 64 * i + 64); ++d) {
        const float x = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, qv[i]), d & 63));
        if (on) dot = fmaf(x, static_cast<float>(k[d]), dot);
      }
    if (on) {
      s = dot * A.scale;
      if constexpr (kI8) {
        const int64_t at = (static_cast<int64_t>(page) * A.c.kv_heads + kv_head) * A.c.page_size + off;
        s *= A.c.k_scale[at];
        vs = A.c.v_scale[at];
      }
      s *= kLog2e;
    }
    float top = on ? fmaxf(s, kLowest) : -INFINITY;
#pragma unroll
    for (int o = 32; o >= 1; o /= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float m1 = fmaxf(R.m, top), ref = m1 == -INFINITY ? 0.0f : m1;
    float p = on ? __builtin_amdgcn_exp2f(s - ref) : 0.0f;
    const float keep = __builtin_amdgcn_exp2f(R.m - ref);  // 0 for the first keys
    float sum = p;
#pragma unroll
    for (int o = 32; o >= 1; o /= 2) sum += __shfl_xor(sum, o, 64);
    R.l = R.l * keep + sum;
    R.m = m1;
    p *= vs;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) R.acc[i] *= keep;
    for (int x = 0; x < n; ++x) {
      if (!__builtin_amdgcn_readlane(on, x)) continue;
      const int64_t pg = __builtin_amdgcn_readlane(page, x), o = __builtin_amdgcn_readlane(off, x);
      const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), x));
      const T* v = static_cast<const T*>(A.c.v) + pg * A.c.v_stride[0] + kv_head * A.c.v_stride[1] + o * A.c.v_stride[2];
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (lane + 64 * i < dim) R.acc[i] = fmaf(w, static_cast<float>(v[lane + 64 * i]), R.acc[i]);
    }
  }
  return R;
}

// The result of a row whose keys are all in.
__device__ __forceinline__ void row_out(const AttnArgs& A, const RowSums& R, int64_t t, int64_t head) {
  const int lane = threadIdx.x & 63;
  const bool none = R.m == -INFINITY;
  __bf16* out = reinterpret_cast<__bf16*>(A.out) + t * A.os[0] + head * A.os[1];
#pragma unroll
  for (int i = 0; i < kOwn; ++i)
    if (lane + 64 * i < A.c.head_dim) out[lane + 64 * i] = static_cast<__bf16>(none ? 0.0f : R.acc[i] / R.l);
  if (A.lse && lane == 0) A.lse[t * A.q_heads + head] = none ? -INFINITY : (R.m + __builtin_amdgcn_logf(R.l)) * kLn2;
}

}  // namespace bitcos_attn
