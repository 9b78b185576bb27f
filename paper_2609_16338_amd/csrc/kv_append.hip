// Storing the new tokens' keys and values in a paged cache: rotation, rounding
// to bfloat16 or to int8 with a scale per (token, head), and the queries
// rotated and rounded to the bfloat16 that the attention reads, in one pass.
//
// Every (token, head) row is read once and written once; the row's absmax and
// the rotation (value i with value i + dim / 2) need only lanes of one wave.
// Bound by memory for prompts and by latency for decode steps.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device_common.h"
#include "kv_common.h"

namespace {

using namespace bitcos_dev;

struct AppendArgs {
  bitcos_kv_cache c;
  const void* x[3];       // q, k, v
  int64_t xs[3][2];       // strides {token, head}
  uint16_t* q_out;
  int64_t qs[2];
  const int32_t* slots;
  const int32_t* positions;
  const float* cos;
  const float* sin;
  int32_t tokens, q_heads, rot, max_pos;
};

// A row's place: which of q, k, v, which head, where it goes.
struct Row {
  int kind;  // 0 q, 1 k, 2 v
  int64_t token;
  int head;
  int32_t slot;  // -1: not stored
  int32_t pos;   // -1: outside the tables
};

__device__ __forceinline__ Row row_of(const AppendArgs& A, int64_t row, int heads) {
  Row R;
  R.token = row / heads;
  int h = static_cast<int>(row - R.token * heads);
  R.kind = h < A.q_heads ? 0 : h < A.q_heads + A.c.kv_heads ? 1 : 2;
  R.head = R.kind == 0 ? h : R.kind == 1 ? h - A.q_heads : h - A.q_heads - A.c.kv_heads;
  R.pos = 0;
  if (A.rot) {
    const int32_t p = A.positions[R.token];
    R.pos = p >= 0 && p < A.max_pos ? p : -1;
  }
  R.slot = 0;
  if (R.kind) {
    const int32_t s = A.slots[R.token];
    R.slot = s >= 0 && s < A.c.pages * A.c.page_size && R.pos >= 0 ? s : -1;
  }
  return R;
}

template <class T>
__device__ __forceinline__ const T* src_of(const AppendArgs& A, const Row& R) {
  return static_cast<const T*>(A.x[R.kind]) + R.token * A.xs[R.kind][0] + R.head * A.xs[R.kind][1];
}

// Element offset of a slot's row in the cache, and its index in the scales.
__device__ __forceinline__ int64_t cache_at(const AppendArgs& A, const Row& R, int64_t& scale_at) {
  const int32_t page = R.slot / A.c.page_size, off = R.slot - page * A.c.page_size;
  scale_at = (static_cast<int64_t>(page) * A.c.kv_heads + R.head) * A.c.page_size + off;
  const int64_t* st = R.kind == 1 ? A.c.k_stride : A.c.v_stride;
  return page * st[0] + R.head * st[1] + off * st[2];
}

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }

// x1 c - x2 s and x2 c + x1 s with every operation rounded by itself, so that
// the stored values are a plain fp32 computation's (the compiler would fuse
// the products into the sums otherwise, for the _rn intrinsics too).
__device__ __forceinline__ void rotate(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float x = a, y = b;
  a = x * c - y * s;
  b = y * c + x * s;
}

// The largest |x| of a row is taken as an integer, which orders infinity behind
// every number and NaN behind infinity; a maximum of floats would drop NaN.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Scale and largest step of a row.  A row with a value that is not finite has
// the scale infinity or NaN and steps of 0: it stands for NaN throughout.
struct RowScale {
  float a, top;
};
__device__ __forceinline__ RowScale row_scale(uint32_t amax) {
  return RowScale{amax == 0 ? 1.0f : __fdiv_rn(__builtin_bit_cast(float, amax), 127.0f), amax < 0x7f800000u ? 127.0f : 0.0f};
}
__device__ __forceinline__ int8_t to_i8(float x, RowScale s) {
  return static_cast<int8_t>(fminf(fmaxf(rintf(__fdiv_rn(x, s.a)), -s.top), s.top));
}

// Any head size, rotation width, stride and alignment: a wave per row, lane l
// has the values l, l + 64, ... of it.  8192 bf16 tokens (32/8 heads) of 128
// values, half of them rotated: 176 us, where a whole rotation takes 35 below
// (inputs that stay in the caches).
template <class T>
__global__ void __launch_bounds__(256) kv_append_general_kernel(AppendArgs A) {
  const int lane = threadIdx.x & 63, heads = A.q_heads + 2 * A.c.kv_heads, dim = A.c.head_dim, half = A.rot / 2;
  const int64_t rows = static_cast<int64_t>(A.tokens) * heads;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); row < rows;
       row += static_cast<int64_t>(gridDim.x) * 4) {
    const Row R = row_of(A, row, heads);
    if (R.kind && R.slot < 0) continue;
    const T* src = src_of<T>(A, R);
    const bool turn = R.kind < 2 && A.rot;
    float v[BITCOS_KV_MAX_DIM / 64];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < BITCOS_KV_MAX_DIM / 64; ++i) {
      const int d = lane + 64 * i;
      v[i] = d < dim ? widen(src[d]) : 0.0f;
      if (turn && d < A.rot && R.pos >= 0) {
        const int j = d < half ? d : d - half;
        const float o = widen(src[d < half ? d + half : d - half]);
        const float c = A.cos[static_cast<int64_t>(R.pos) * half + j], s = A.sin[static_cast<int64_t>(R.pos) * half + j];
        float lo = d < half ? v[i] : o, hi = d < half ? o : v[i];
        rotate(lo, hi, c, s);
        v[i] = d < half ? lo : hi;
      }
      amax = max(amax, abs_bits(v[i]));
    }
    if (R.kind == 0) {
      __bf16* dst = reinterpret_cast<__bf16*>(A.q_out) + R.token * A.qs[0] + R.head * A.qs[1];
#pragma unroll
      for (int i = 0; i < BITCOS_KV_MAX_DIM / 64; ++i)
        if (lane + 64 * i < dim) dst[lane + 64 * i] = static_cast<__bf16>(R.pos < 0 ? 0.0f : v[i]);
      continue;
    }
    int64_t scale_at;
    const int64_t at = cache_at(A, R, scale_at);
    void* base = R.kind == 1 ? A.c.k : A.c.v;
    if (A.c.dtype == BITCOS_KV_BF16) {
#pragma unroll
      for (int i = 0; i < BITCOS_KV_MAX_DIM / 64; ++i)
        if (lane + 64 * i < dim) static_cast<__bf16*>(base)[at + lane + 64 * i] = static_cast<__bf16>(v[i]);
    } else {
#pragma unroll
      for (int o = 32; o >= 1; o /= 2) amax = max(amax, __shfl_xor(amax, o, 64));
      const RowScale scale = row_scale(amax);
#pragma unroll
      for (int i = 0; i < BITCOS_KV_MAX_DIM / 64; ++i)
        if (lane + 64 * i < dim) static_cast<int8_t*>(base)[at + lane + 64 * i] = to_i8(v[i], scale);
      if (lane == 0) (R.kind == 1 ? A.c.k_scale : A.c.v_scale)[scale_at] = scale.a;
    }
  }
}

// kPer values a lane from each half of the head, so that a value and its
// partner in the rotation share a lane and an access of the inputs is 16 bytes
// (bfloat16: eight values; fp32: four): heads of 64, 128 and 256 values,
// rotated as a whole or not at all, on 16-byte boundaries.  D / (2 kPer) lanes
// have a row.  8192 bf16 tokens (32/8 heads, 206 MB): 40.7 us, 5.1 TB/s (a
// large copy: 4.8), into int8 46; with four values a lane, 8-byte reads, 57 us.  45 tokens of
// fp32 into int8: 3.8 us, one token: 2.6 us, the launch and two dependent reads.
template <class T, int D, bool kI8>
__global__ void __launch_bounds__(256) kv_append_kernel(AppendArgs A) {
  constexpr int kPer = 16 / sizeof(T), kLanes = D / (2 * kPer), kHalf = D / 2;
  typedef float f32xn __attribute__((ext_vector_type(kPer), aligned(16)));
  typedef __bf16 bf16xn __attribute__((ext_vector_type(kPer)));
  typedef int8_t i8xn __attribute__((ext_vector_type(kPer)));
  typedef T srcn __attribute__((ext_vector_type(kPer)));
  const int heads = A.q_heads + 2 * A.c.kv_heads, j = threadIdx.x % kLanes;
  const int64_t rows = static_cast<int64_t>(A.tokens) * heads;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
  if (row >= rows) return;  // whole rows: the lanes that exchange values stay together
  const Row R = row_of(A, row, heads);
  if (R.kind && R.slot < 0) return;
  const T* src = src_of<T>(A, R) + kPer * j;
  const srcn ra = *reinterpret_cast<const srcn*>(src), rb = *reinterpret_cast<const srcn*>(src + kHalf);
  const bool turn = R.kind < 2 && A.rot && R.pos >= 0;
  f32xn c, s;
  if (turn) {
    c = *reinterpret_cast<const f32xn*>(A.cos + static_cast<int64_t>(R.pos) * kHalf + kPer * j);
    s = *reinterpret_cast<const f32xn*>(A.sin + static_cast<int64_t>(R.pos) * kHalf + kPer * j);
  }
  float a[kPer], b[kPer];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    a[i] = widen(ra[i]);
    b[i] = widen(rb[i]);
    if (turn) rotate(a[i], b[i], c[i], s[i]);
    amax = max(amax, max(abs_bits(a[i]), abs_bits(b[i])));
  }
  bf16xn wa, wb;
#pragma unroll
  for (int i = 0; i < kPer; ++i) wa[i] = static_cast<__bf16>(a[i]), wb[i] = static_cast<__bf16>(b[i]);
  if (R.kind == 0) {
    uint16_t* dst = A.q_out + R.token * A.qs[0] + R.head * A.qs[1] + kPer * j;
    if (R.pos < 0) wa = wb = bf16xn{};
    *reinterpret_cast<bf16xn*>(dst) = wa;
    *reinterpret_cast<bf16xn*>(dst + kHalf) = wb;
    return;
  }
  int64_t scale_at;
  const int64_t at = cache_at(A, R, scale_at) + kPer * j;
  void* base = R.kind == 1 ? A.c.k : A.c.v;
  if constexpr (!kI8) {
    *reinterpret_cast<bf16xn*>(static_cast<uint16_t*>(base) + at) = wa;
    *reinterpret_cast<bf16xn*>(static_cast<uint16_t*>(base) + at + kHalf) = wb;
  } else {
#pragma unroll
    for (int o = kLanes / 2; o >= 1; o /= 2) amax = max(amax, __shfl_xor(amax, o, 64));
    const RowScale scale = row_scale(amax);
    i8xn pa, pb;
#pragma unroll
    for (int i = 0; i < kPer; ++i) pa[i] = to_i8(a[i], scale), pb[i] = to_i8(b[i], scale);
    *reinterpret_cast<i8xn*>(static_cast<int8_t*>(base) + at) = pa;
    *reinterpret_cast<i8xn*>(static_cast<int8_t*>(base) + at + kHalf) = pb;
    if (j == 0) (R.kind == 1 ? A.c.k_scale : A.c.v_scale)[scale_at] = scale.a;
  }
}

template <int D>
auto vector_kernel(bool f32, bool i8) {
  return f32 ? (i8 ? kv_append_kernel<float, D, true> : kv_append_kernel<float, D, false>)
             : (i8 ? kv_append_kernel<__bf16, D, true> : kv_append_kernel<__bf16, D, false>);
}

}  // namespace

extern "C" int bitcos_kv_append(const bitcos_kv_cache* cache, int32_t tokens, int32_t act_dtype, const void* k,
                                const int64_t* k_stride, const void* v, const int64_t* v_stride, const int32_t* slots,
                                int32_t q_heads, const void* q, const int64_t* q_stride, void* q_out,
                                const int64_t* q_out_stride, int32_t rot_dim, const float* cos, const float* sin,
                                int32_t max_pos, const int32_t* positions, void* stream) {
  if (const int st = kv_cache_status(cache)) return st;
  if (!k || !v || !k_stride || !v_stride || !slots || tokens < 1) return BITCOS_E_ARG;
  if (act_dtype != BITCOS_ACT_F32 && act_dtype != BITCOS_ACT_BF16) return BITCOS_E_ARG;
  if (q ? q_heads < 1 || !q_stride || !q_out || !q_out_stride : q_heads != 0) return BITCOS_E_ARG;
  if (rot_dim < 0 || rot_dim % 2 || rot_dim > cache->head_dim) return BITCOS_E_ARG;
  if (rot_dim && (!cos || !sin || !positions || max_pos < 1)) return BITCOS_E_ARG;
  AppendArgs A{};
  A.c = *cache;
  A.x[0] = q;
  A.x[1] = k;
  A.x[2] = v;
  for (int i = 0; i < 2; ++i) {
    A.xs[0][i] = q ? q_stride[i] : 0;
    A.xs[1][i] = k_stride[i];
    A.xs[2][i] = v_stride[i];
    A.qs[i] = q ? q_out_stride[i] : 0;
    if (A.xs[0][i] < 0 || A.xs[1][i] < 0 || A.xs[2][i] < 0 || A.qs[i] < 0) return BITCOS_E_ARG;
  }
  A.q_out = static_cast<uint16_t*>(q_out);
  A.slots = slots;
  A.positions = positions;
  A.cos = cos;
  A.sin = sin;
  A.tokens = tokens;
  A.q_heads = q ? q_heads : 0;
  A.rot = rot_dim;
  A.max_pos = max_pos;
  const int64_t rows = static_cast<int64_t>(tokens) * (A.q_heads + 2ll * cache->kv_heads);
  const int dim = cache->head_dim, in = act_dtype == BITCOS_ACT_F32 ? 4 : 2, elem = cache->dtype == BITCOS_KV_I8 ? 1 : 2;
  const bool whole = rot_dim == 0 || (rot_dim == dim && reinterpret_cast<uintptr_t>(cos) % 16 == 0 && reinterpret_cast<uintptr_t>(sin) % 16 == 0);
  if ((dim == 64 || dim == 128 || dim == 256) && whole && rows_aligned16(q, A.xs[0], 2, in) && rows_aligned16(k, k_stride, 2, in) &&
      rows_aligned16(v, v_stride, 2, in) && rows_aligned16(q_out, A.qs, 2, 2) && rows_aligned16(cache->k, cache->k_stride, 3, elem) &&
      rows_aligned16(cache->v, cache->v_stride, 3, elem)) {
    const bool f32 = act_dtype == BITCOS_ACT_F32, i8 = cache->dtype == BITCOS_KV_I8;
    const auto fn = dim == 64 ? vector_kernel<64>(f32, i8) : dim == 128 ? vector_kernel<128>(f32, i8) : vector_kernel<256>(f32, i8);
    const int64_t per = 256 * 2 * (16 / in) / dim, blocks = (rows + per - 1) / per;
    // A launch holds fewer than 2^32 threads: one of more fails, or starts with the count's low 32 bits, with no error.
    if (blocks * 256 <= UINT32_MAX) {
      hipLaunchKernelGGL(fn, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), A);
      return bitcos_launch_status();
    }
  }
  const int64_t blocks = std::min<int64_t>((rows + 3) / 4, 65536);
  const auto fn = act_dtype == BITCOS_ACT_F32 ? kv_append_general_kernel<float> : kv_append_general_kernel<__bf16>;
  hipLaunchKernelGGL(fn, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), A);
  return bitcos_launch_status();
}
