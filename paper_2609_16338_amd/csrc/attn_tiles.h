// Pieces of the matrix-core attention kernels: copies of key and value rows
// into LDS, operand types, and what a lane does with a row's scores.
#pragma once

#include "attn_rows.h"
#include "attn_schedule.h"

namespace bitcos_attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* lds_ptr;

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)(p)));
}

// A buffer resource: `bytes` bytes from base; reads past them give zeros.
__device__ __forceinline__ u32x4 raw_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const auto uni = [](uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))); };
  return u32x4{uni(static_cast<uint32_t>(a)), uni(static_cast<uint32_t>(a >> 32) & 0xFFFFu), uni(bytes), 0x00020000u};
}

// Copies 16 (4) bytes per lane from r + voff[i] straight into LDS, lane after
// lane from `lds` + 1024 i on; zeros where the resource ends.  Written as
// assembly because the compiler would wait for every such copy before any LDS
// read; here each wait is counted by hand.  There is no register to return to,
// and the reads of what the copies overwrite are over (lgkmcnt 0) before they
// start.  The s_nop cover the hazards that the compiler does not see inside:
// a scalar register written by a vector instruction (5 states), and M0 written
// just before (1).  `once`: the bytes are read by nobody else, so they need
// not stay in the caches (64 requests over 800 MB of bfloat16: 161 us without,
// 144 us with it).
#define ATTN_COPY(HINT)                                                                                                          \
  if constexpr (N == 1)                                                                                                          \
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen " HINT "lds" ::"s"(lds), "v"(voff[0]), "s"(r) \
                 : "memory");                                                                                                    \
  else if constexpr (N == 2)                                                                                                     \
    asm volatile(                                                                                                                \
        "s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %3, 0 offen " HINT                                               \
        "lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen " HINT "lds" ::"s"(lds),               \
        "v"(voff[0]), "v"(voff[1]), "s"(r)                                                                                       \
        : "memory", "scc");                                                                                                      \
  else                                                                                                                           \
    asm volatile(                                                                                                                \
        "s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %5, 0 offen " HINT                                               \
        "lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen " HINT                                \
        "lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen " HINT                                \
        "lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen " HINT "lds" ::"s"(lds),               \
        "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(r)                                                           \
        : "memory", "scc")
template <bool once, int N>
__device__ __forceinline__ void copy16(u32x4 r, const uint32_t (&voff)[N], uint32_t lds) {
  static_assert(N == 1 || N == 2 || N == 4, "copies of 16 rows");
  if constexpr (once) {
    ATTN_COPY("nt ");
  } else {
    ATTN_COPY("");
  }
}
#undef ATTN_COPY
__device__ __forceinline__ void copy4(u32x4 r, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(r) : "memory");
}
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// At most N of the wave's vector-memory accesses still under way.
template <int N>
__device__ __forceinline__ void copies_left() {
  static_assert(N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// Value of the larger of lane l's and of lanes l ^ 16, l ^ 32, l ^ 48's, and the sum of the four.
__device__ __forceinline__ float as_float(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float max_groups(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(as_uint(v), as_uint(v), false, false);
  v = fmaxf(as_float(p[0]), as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane16_swap(as_uint(v), as_uint(v), false, false);
  return fmaxf(as_float(q[0]), as_float(q[1]));
}
__device__ __forceinline__ float sum_groups(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(as_uint(v), as_uint(v), false, false);
  v = as_float(p[0]) + as_float(p[1]);
  const auto q = __builtin_amdgcn_permlane16_swap(as_uint(v), as_uint(v), false, false);
  return as_float(q[0]) + as_float(q[1]);
}

// Eight int8 values (two dwords) as bfloat16: exact.  A byte converts in one
// instruction (sub-dword access, sign extended); the compiler would shift the
// odd bytes down first.
template <int kByte>
__device__ __forceinline__ float byte_float(uint32_t v) {
  float f;
  if constexpr (kByte == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(v));
  if constexpr (kByte == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(v));
  if constexpr (kByte == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(v));
  if constexpr (kByte == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(v));
  return f;
}
__device__ __forceinline__ bf16x8 widen8(u32x2 v) {
  bf16x8 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    o[4 * i] = static_cast<__bf16>(byte_float<0>(v[i]));
    o[4 * i + 1] = static_cast<__bf16>(byte_float<1>(v[i]));
    o[4 * i + 2] = static_cast<__bf16>(byte_float<2>(v[i]));
    o[4 * i + 3] = static_cast<__bf16>(byte_float<3>(v[i]));
  }
  return o;
}

// Whether a row of the item's token `tok` that sees some of keys [from, to) ended with the maximum of none: all their
// scores are -infinity, or their pages are none of the cache's.  Which of the two, rows_again finds out (slowly: not asked
// for tiles without a page of the cache's, which a table may have many of).
__device__ __forceinline__ bool nothing_seen(const AttnArgs& A, const Item& I, int tok, float m, int from, int to) {
  int lo, hi;
  seen(A, I.s, I.first + tok, lo, hi);
  return m == -INFINITY && min(hi, to) > max(lo, from);
}

// Infinite and NaN values (or scales): in the products a weight of zero (a row
// that does not see the key) would make NaN of them, and a weight in two halves, of which
// the lower may be zero or negative, NaN of an infinity.  Either leaves a sum
// that is not finite, and stays; so the rows of an item whose sums end up so
// (or that saw nothing but scores of -infinity, above, or huge ones) are done
// again one by one, over the keys that each sees of keys [from, to).
template <class T, int D>
__device__ __forceinline__ void rows_again(const AttnArgs& A, const Parts& P, const Item& I, int me, int slot, bool whole, int from, int to,
                                           int row0, int row1) {
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int row = row0; row < row1; ++row) {
    const int tok = static_cast<int>(row * A.group_inv >> 16);
    const int64_t t = I.s.q0 + I.first + tok, head = static_cast<int64_t>(I.h) * A.group + row - tok * A.group;
    int lo, hi;
    seen(A, I.s, I.first + tok, lo, hi);
    const RowSums R = row_over_keys<T>(A, I.r, t, head, I.h, max(lo, from), min(hi, to));
    if (whole) {
      row_out(A, R, t, head);
      continue;
    }
    const int64_t at = (static_cast<int64_t>(me) * 2 + slot) * P.rows + row;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) P.acc[at * D + lane + 64 * i] = R.acc[i];
    if (lane == 0) {
      P.ml[2 * at] = R.m;
      P.ml[2 * at + 1] = R.l;
    }
  }
}

}  // namespace bitcos_attn
