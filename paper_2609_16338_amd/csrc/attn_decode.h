// Attention of few query rows per request and kv head (single tokens, drafted
// tokens) over a paged cache, on the matrix cores.
//
// What bounds it is reading keys and values once: 2 dim values per key and kv
// head against 4 dim flops per query row, far below the matrix cores' rate at
// up to 64 rows.  So the kernel is built to keep copies in flight.  A wave is
// a worker of its own (64 threads a workgroup, no barrier anywhere): it copies
// 32 keys and 32 values of one kv head into LDS (buffer loads straight to LDS,
// 16 bytes a lane), multiplies the keys by all of its query rows, starts the
// copy of the next keys, turns the scores into weights, multiplies the values
// by them and starts the copy of the next values.  A tile of bfloat16 keys and
// values of 128 is 16 KB, so eight waves a CU hold 128 KB of its 160 KB of LDS,
// each with one to two copies under way.
//
// Measured with its join, 128 values a head: 64 requests of 100 to 16384 keys
// (32/8 heads, bfloat16, 801 MB) 137 us, 5.9 TB/s; 32 of up to 131072 (int8,
// 1.84 GB) 293 us, 6.3 TB/s; a plain streaming read reaches 6.1 TB/s here.  No
// LDS bank conflict; the vector units issue for 14% (int8: 53%) of the cycles.
// One sequence of 2000 keys: 12.0 us, of which 7 are this kernel (finding its
// place, the page ids, one tile: three dependent trips to memory) and 4.5 the join.
//
// Scores stand transposed, S^T = K Q^T (16 keys x 16 rows an MFMA): a lane then
// holds one row's scores of keys 4g .. 4g + 3 (g = lane / 16), the row maximum
// is a maximum over registers and two lane exchanges, and the weights are
// already where the product O^T = V^T P^T wants its right operand, if that
// product takes its 32 keys in the order that the lanes hold them: slot 8g + j
// is key 4g + j for j < 4, key 16 + 4g + j - 4 for the others.  Values are
// read transposed from LDS in that order.
//
// LDS holds rows as they come, but 16-byte chunk c of row r stands at chunk
// c ^ f(r) (each lane copies the chunk that belongs in its place), with f such
// that the lanes of one LDS pass touch every bank once: for keys 16 rows of one
// chunk, for values 8 rows of two chunks (16 rows of one, int8).
//
// The weights are rounded to bfloat16 twice over, p = hi + lo, and both halves
// multiplied: the second product is free where memory is what bounds, and the
// result is as exact as fp32 weights would make it.
#pragma once

#include <type_traits>

#include "attn_tiles.h"

namespace bitcos_attn {

template <int D, bool kI8, int NT>
struct DecodeTile {
  static constexpr int kKeys = 32;
  static constexpr int kRow = D * (kI8 ? 1 : 2);      // bytes
  static constexpr int kChunks = kRow / 16;           // per row
  static constexpr int kRowsPerCopy = 64 / kChunks;   // rows that one copy brings
  static constexpr int kCopies = 16 / kRowsPerCopy;   // per half tile (16 keys)
  static constexpr int kPending = 2 * kCopies + (kI8 ? 2 : 0);  // per tile of keys, and of values
  static constexpr int kRows = 16 * NT;
  static constexpr int kLds = 2 * kKeys * kRow + (kI8 ? 4 * 256 : 0);

  // Chunk permutations of row r (0..31).
  __device__ static __forceinline__ int fk(int r) { return (r / (16 / kChunks)) & (kChunks - 1); }
  __device__ static __forceinline__ int fv(int r) {
    if constexpr (!kI8) return kChunks == 16 ? 2 * (r & 7) : 2 * ((r >> 1) & 3);
    return kChunks == 8 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 2) & 1) | ((r >> 4) & 1) << 1;
  }
};

// The rows of 16 keys, which lie in one page: resources of keys and values (and
// scales) that end behind the last key that any query sees.  (Rows before the
// first are read as they are.)
struct Half {
  u32x4 k, v, ks, vs;
};

// Two waves a SIMD, no more: left to themselves the 2048 workgroups do not spread evenly, a SIMD getting three and
// another one, as the launch before happens to leave things (32 long int8 requests: 324 us so, 293 us spread).
template <int D, bool kI8, int NT>
__global__ void __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 2)))
paged_attn_decode_kernel(AttnArgs, Parts P, int most, int least_log2) {
  using T = DecodeTile<D, kI8, NT>;
  using Value = std::conditional_t<kI8, int8_t, __bf16>;
  constexpr int kSteps = D / 32, kOut = D / 16, kElem = kI8 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) char s_k[T::kKeys * T::kRow];
  __shared__ __attribute__((aligned(1024))) char s_v[T::kKeys * T::kRow];
  __shared__ __attribute__((aligned(256))) float s_scale[kI8 ? 4 * 64 : 4];  // keys 0-15, 16-31, values 0-15, 16-31
  const int lane = threadIdx.x, c = lane & 15, g = lane >> 4;
  const int me = blockIdx.x;
  Schedule<T::kKeys> sched;
  int64_t u, u1;
  Item I;
  int at;
  if (!sched.start(args_anew(), me, most, least_log2, u, u1, I, at)) {
    if (lane == 0) P.note[me] = int4{-1, 0, 0, 0};
    return;
  }
  // Where each lane's chunk of a copy comes from (bytes from the half's first row), for keys and values.
  uint32_t kfrom[2][T::kCopies], vfrom[2][T::kCopies], kts, vts, page_mask;
  float mul;
  {
    const AttnArgs& A = args_anew();
    kts = static_cast<uint32_t>(A.c.k_stride[2]) * kElem;
    vts = static_cast<uint32_t>(A.c.v_stride[2]) * kElem;
    page_mask = A.c.page_size - 1;
    mul = A.scale * kLog2e;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int i = 0; i < T::kCopies; ++i) {
        const int row = i * T::kRowsPerCopy + lane / T::kChunks, ch = lane % T::kChunks;
        kfrom[hf][i] = row * kts + 16 * (ch ^ T::fk(16 * hf + row));
        vfrom[hf][i] = row * vts + 16 * (ch ^ T::fv(16 * hf + row));
      }
  }
  const uint32_t lk = lds_addr(s_k), lv = lds_addr(s_v), lsc = lds_addr(s_scale);
  bool noted = false;

  while (u < u1) {
    const int k0 = at, k1 = static_cast<int>(min(static_cast<int64_t>(I.units), k0 + (u1 - u)));
    // The page ids of 64 half tiles, a lane each (-1: names no page, or no query sees its keys), read together and waited
    // for here: one read for every tile would be waited for in every tile.
    int ids = 0, ids_from = 0;
    bool named = false;  // a page of this worker's tiles is one of the cache's
    const auto read_ids = [&](int kt) {
      const AttnArgs& A = args_anew();
      const int32_t* trow = A.table + static_cast<int64_t>(I.r) * A.width;
      ids_from = kt;
      const int key0 = 32 * (I.t0 + kt) + 16 * lane;
      ids = key0 < I.hi && key0 + 16 > I.lo ? trow[key0 >> A.page_shift] : -1;
      wait_vmem_all();
      if (ids >= A.c.pages) ids = -1;
      named |= __any(ids >= 0 && kt + lane / 2 < k1);
    };
    // Where the item's keys and values lie (kv head h of page 0), bytes from page to page, and of the scales.
    const char *kbase, *vbase, *ksbase, *vsbase;
    uint32_t kps, vps, sps;
    // Resources of half `hf` of the item's key tile kt; false where its page id names no page.
    const auto half_of = [&](int kt, int hf, Half& H) -> bool {
      const int key0 = 32 * (I.t0 + kt) + 16 * hf;
      const int id = __builtin_amdgcn_readlane(ids, 2 * (kt - ids_from) + hf);  // (a lane past the last: not copied)
      const uint32_t page = max(id, 0), off = key0 & page_mask;
      const int n = id < 0 || kt >= k1 ? 0 : max(0, min(16, I.hi - key0));
      H.k = raw_rsrc(kbase + static_cast<uint64_t>(page) * kps + off * kts, n ? (n - 1) * kts + T::kRow : 0);
      H.v = raw_rsrc(vbase + static_cast<uint64_t>(page) * vps + off * vts, n ? (n - 1) * vts + T::kRow : 0);
      if constexpr (kI8) {
        H.ks = raw_rsrc(ksbase + static_cast<uint64_t>(page) * sps + off * 4, 4 * n);
        H.vs = raw_rsrc(vsbase + static_cast<uint64_t>(page) * sps + off * 4, 4 * n);
      }
      return id >= 0;
    };
    const auto copy_keys = [&](const Half (&H)[2]) {
      lds_reads_done();
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        copy16<true>(H[hf].k, kfrom[hf], lk + hf * 16 * T::kRow);
        if constexpr (kI8) copy4(H[hf].ks, lane * 4, lsc + 256 * hf);
      }
    };
    const auto copy_values = [&](const Half (&H)[2]) {
      lds_reads_done();
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        copy16<true>(H[hf].v, vfrom[hf], lv + hf * 16 * T::kRow);
        if constexpr (kI8) copy4(H[hf].vs, lane * 4, lsc + 512 + 256 * hf);
      }
    };

    bool ok[2];
    int rows, rlo[NT], rhi[NT], all_lo, all_hi;  // rows of the item; the keys that each sees, that all see
    // Queries: lane (c, g) has row 16 nt + c's values of each 32-value step, 8 at 8g (int8: 16 at 16g of each 64).
    bf16x8 q[NT][kSteps];
    {
      const AttnArgs& A = args_anew();
      kbase = static_cast<const char*>(A.c.k) + kElem * I.h * A.c.k_stride[1];
      vbase = static_cast<const char*>(A.c.v) + kElem * I.h * A.c.v_stride[1];
      kps = static_cast<uint32_t>(kElem * A.c.k_stride[0]);
      vps = static_cast<uint32_t>(kElem * A.c.v_stride[0]);
      ksbase = reinterpret_cast<const char*>(A.c.k_scale + static_cast<int64_t>(I.h) * A.c.page_size);
      vsbase = reinterpret_cast<const char*>(A.c.v_scale + static_cast<int64_t>(I.h) * A.c.page_size);
      sps = 4u * A.c.kv_heads * A.c.page_size;
      read_ids(k0);
      Half H[2];
      ok[0] = half_of(k0, 0, H[0]);
      ok[1] = half_of(k0, 1, H[1]);
      copy_keys(H);
      copy_values(H);
      rows = I.count * A.group;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = 16 * nt + c;
        const int tok = static_cast<int>(row * A.group_inv >> 16), head = row - tok * A.group;
        const bool on = row < rows;
        const int64_t t = I.s.q0 + I.first + tok, hq = static_cast<int64_t>(I.h) * A.group + head;
        seen(A, I.s, I.first + tok, rlo[nt], rhi[nt]);
        if (!on || rhi[nt] < rlo[nt]) rlo[nt] = rhi[nt] = 0;
        const uint16_t* src = A.q + t * A.qs[0] + hq * A.qs[1];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int d = kI8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
          u32x4 w{0, 0, 0, 0};
          if (on) w = *reinterpret_cast<const u32x4*>(src + d);
          q[nt][s] = __builtin_bit_cast(bf16x8, w);
        }
      }
      int x;
      seen(A, I.s, I.first, x, all_hi);
      seen(A, I.s, I.first + I.count - 1, all_lo, x);
    }
    // The queries are there before the loop: a wait for them inside it
    // would be one for every copy under way.
    wait_vmem_all();
    f32x4 acc[NT][kOut];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt] = -INFINITY;
      l[nt] = 0.0f;
#pragma unroll
      for (int o = 0; o < kOut; ++o) acc[nt][o] = f32x4{0, 0, 0, 0};
    }
    for (int kt = k0; kt < k1; ++kt) {
      const int key0 = 32 * (I.t0 + kt);
      const bool bad0 = !ok[0], bad1 = !ok[1];
      const bool edge = key0 < all_lo || key0 + 32 > all_hi || bad0 || bad1;
      Half N[2];
      if (kt + 1 - ids_from == 32 && kt + 1 < k1) read_ids(kt + 1);
      ok[0] = half_of(kt + 1, 0, N[0]);  // past the last tile: nothing but zeros
      ok[1] = half_of(kt + 1, 1, N[1]);
      copies_left<T::kPending>();
      f32x4 s[NT][2];
      f32x4 kscale[2], vscale[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][hf] = f32x4{0, 0, 0, 0};
        const int row = 16 * hf + c;
        if constexpr (kI8) {
          kscale[hf] = *reinterpret_cast<const f32x4*>(&s_scale[64 * hf + 4 * g]);
#pragma unroll
          for (int s2 = 0; s2 < kSteps / 2; ++s2) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(s_k + row * T::kRow + 16 * ((4 * s2 + g) ^ T::fk(row)));
            const bf16x8 a = widen8(u32x2{w[0], w[1]}), b = widen8(u32x2{w[2], w[3]});
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              s[nt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[nt][2 * s2], s[nt][hf], 0, 0, 0);
              s[nt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, q[nt][2 * s2 + 1], s[nt][hf], 0, 0, 0);
            }
          }
        } else {
#pragma unroll
          for (int st = 0; st < kSteps; ++st) {
            const bf16x8 a = *reinterpret_cast<const bf16x8*>(s_k + row * T::kRow + 16 * ((4 * st + g) ^ T::fk(row)));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[nt][st], s[nt][hf], 0, 0, 0);
          }
        }
      }
      copy_keys(N);
      // Whether row 16 nt + c does not see the lane's key i (of eight).
      const auto unseen = [&](int nt, int i) {
        const int key = key0 + 16 * (i / 4) + 4 * g + i % 4;
        return static_cast<uint32_t>(key - rlo[nt]) >= static_cast<uint32_t>(rhi[nt] - rlo[nt]) || (i < 4 ? bad0 : bad1);
      };
      // Scores to weights.
      bf16x8 hi[NT], lo[NT];
      float keep[NT];
      bool moved = false;
      copies_left<T::kPending>();  // the values are there
      if constexpr (kI8) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) vscale[hf] = *reinterpret_cast<const f32x4*>(&s_scale[128 + 64 * hf + 4 * g]);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float w[8];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = s[nt][i / 4][i % 4] * mul;
          if constexpr (kI8) w[i] *= kscale[i / 4][i % 4];
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = unseen(nt, i) ? -INFINITY : w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, w[i]);
        top = max_groups(top);
        const float m1 = fmaxf(m[nt], top), ref = m1 == -INFINITY ? 0.0f : m1;
        keep[nt] = __builtin_amdgcn_exp2f(m[nt] - ref);
        moved |= m1 != m[nt];
        m[nt] = m1;
        float sum = 0.0f, p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(w[i] - ref);
          sum += p[i];
          if constexpr (kI8) p[i] *= vscale[i / 4][i % 4];
        }
        if (kI8 && edge) {  // the scale of a key not seen may be anything
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = unseen(nt, i) ? 0.0f : p[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          hi[nt][i] = static_cast<__bf16>(p[i]);
          lo[nt][i] = static_cast<__bf16>(p[i] - static_cast<float>(hi[nt][i]));
        }
        l[nt] = l[nt] * keep[nt] + sum;
      }
      if (__any(moved)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int o = 0; o < kOut; ++o) acc[nt][o] *= keep[nt];
      }
#pragma unroll
      for (int o = 0; o < kOut; ++o) {
        bf16x8 a;
        if constexpr (kI8) {
          const int row = (c < 8 ? 0 : 12) + 4 * g + c / 2;
          const char* p = s_v + row * T::kRow + 16 * (o ^ T::fv(row)) + 8 * (c & 1);
          a = widen8(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p)));
        } else {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int row = 16 * hf + 4 * g + c / 4;
            const char* p = s_v + row * T::kRow + 16 * ((2 * o + (c & 3) / 2) ^ T::fv(row)) + 8 * (c & 1);
            const bf16x4 w = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p));
#pragma unroll
            for (int i = 0; i < 4; ++i) a[4 * hf + i] = w[i];
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hi[nt], acc[nt][o], 0, 0, 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, lo[nt], acc[nt][o], 0, 0, 0);
      }
      copy_values(N);
    }
    lds_reads_done();
    copies_left<0>();  // the copies past the last tile, before LDS is filled anew
    const AttnArgs& A = args_anew();
    const bool whole = k0 == 0 && k1 == I.units;
    const int slot = k0 > 0 ? kHead : kTail;
    float* pacc = P.acc + (static_cast<int64_t>(me) * 2 + slot) * P.rows * D;
    float* pml = P.ml + (static_cast<int64_t>(me) * 2 + slot) * P.rows * 2;
    bool odd = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 16 * nt + c;
      odd |= named && row < rows && nothing_seen(A, I, static_cast<int>(row * A.group_inv >> 16), m[nt], 32 * (I.t0 + k0), 32 * (I.t0 + k1));
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= !__builtin_isfinite(acc[nt][o][i]);
    }
    odd = __any(odd);
    if (odd) rows_again<Value, D>(A, P, I, me, slot, whole, 32 * (I.t0 + k0), 32 * (I.t0 + k1), 0, rows);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float sum = sum_groups(l[nt]);
      const int row = 16 * nt + c;
      if (row >= rows || odd) continue;
      if (whole) {
        const bool none = m[nt] == -INFINITY && sum == 0.0f;
        const float inv = none ? 0.0f : 1.0f / sum;
        const int tok = static_cast<int>(row * A.group_inv >> 16);
        const int64_t t = I.s.q0 + I.first + tok, hq = static_cast<int64_t>(I.h) * A.group + row - tok * A.group;
        uint16_t* dst = A.out + t * A.os[0] + hq * A.os[1];
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
          bf16x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = static_cast<__bf16>(none ? 0.0f : acc[nt][o][i] * inv);
          *reinterpret_cast<u32x2*>(dst + 16 * o + 4 * g) = __builtin_bit_cast(u32x2, w);
        }
        if (A.lse && g == 0) A.lse[t * A.q_heads + hq] = none ? -INFINITY : (m[nt] + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
#pragma unroll
        for (int o = 0; o < kOut; ++o) *reinterpret_cast<f32x4*>(pacc + row * D + 16 * o + 4 * g) = acc[nt][o];
        if (g == 0) {
          pml[2 * row] = m[nt];
          pml[2 * row + 1] = sum;
        }
      }
    }
    if (k1 < I.units) {
      noted = true;
      if (lane == 0) P.note[me] = sched.note(I, u, k0, rows);
    }
    u += k1 - k0;
    at = 0;
    if (u < u1 && !sched.next(A, I)) break;
  }
  if (!noted && lane == 0) P.note[me] = int4{-1, 0, 0, 0};
}

}  // namespace bitcos_attn
