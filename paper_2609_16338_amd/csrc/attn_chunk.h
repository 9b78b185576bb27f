// Attention of many query rows per request and kv head (chunks of a prompt)
// over a paged cache, on the matrix cores.
//
// What bounds it is multiplying: 4 dim flops per row and visible key.  A
// workgroup of four waves is a worker: its item has up to 128 rows (tokens
// times the query heads of a kv head, so a key tile read once serves all of
// them), 32 a wave, which stay in registers with their sums; keys and values
// pass by in tiles of 64, through LDS in two buffers, the next tile copied
// while the present one is multiplied.  Two workgroups share a CU: while one's
// waves turn scores into weights the other's keep the matrix cores busy (one
// workgroup alone takes 1.4 times as long).  32 rows a wave are what 256
// registers hold; 64 with 512 of them, one wave a SIMD, leave nothing to run
// while scores become weights (799 us against 643 for the prompt below), and
// 32-key tiles for three workgroups a CU spill (839 us).
//
// Measured with its join, 128 values a head, on two cards: a prompt of 8192
// (32/8 heads, bfloat16) 642 and 662 us, 857 and 831 TFLOP/s; 1000 queries after
// 30000 int8 keys (40/8 heads) 816 and 838 us, 766 and 746 TFLOP/s (the first ten
// launches of a burst up to 1070 us each); a library product of 16384 x 16384
// matrices reaches 1363 TFLOP/s.  The matrix cores are busy for 50% (int8: 37%)
// of the cycles, vector instructions issue for 49% (61%): between them all of
// the time, so the two hardly overlap, though a product leaves the vector unit
// half its cycles.  A wave issues for 45% of its time, waits for its turn to
// issue for 36%, for data for 19%.  Without the copies the prompt would take
// 535 us, without either product 446, without the exponentials 580.
//
// Weights multiply the values as one bfloat16, which is off by up to 2^-8 of
// each where the few-row kernel's two halves lose 2^-16: a whole output's error
// is 0.0022 so, 0.0017 (the result's own rounding) with both.  The second
// product would be half of this kernel's matrix work again; for requests
// of few queries alone, beside a chunk, it fits the registers at bfloat16 and
// spills 14 to 57 of them at int8.
//
// As for few rows, scores stand transposed (S^T = K Q^T, 32 keys x 32 rows an
// MFMA): lane l has row l % 32's scores of keys 8 a + 4 h + b (h = l / 32, a =
// 0..3, b = 0..3), needs one lane exchange for the row's maximum, and holds
// the weights where O^T = V^T P^T wants its right operand: of 16 keys, slot
// 8 h + j is key 4 h + j for j < 4, key 8 + 4 h + j - 4 for the others.
// Chunk c of row r stands at chunk c ^ f(r) in LDS, so that the 16 rows of one
// chunk (keys) and 4 rows of four chunks (values) of an LDS pass touch every
// bank once (int8: and the eight chunks of a pass that writes; ChunkTile).
//
// An int8 cache is widened to bfloat16 (exact) on its way into LDS, once for
// the four waves; the scales multiply scores and weights.
#pragma once

#include <type_traits>

#include "attn_tiles.h"

namespace bitcos_attn {

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

template <int D, bool kI8>
struct ChunkTile {
  static constexpr int kKeys = 64, kRows = 128;
  static constexpr int kRow = 2 * D;           // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kBytes = kKeys * kRow;  // of a tile of keys, or of values
  // Chunk c + low (low within c's alignment) of row r stands at at(c, low) ^ f(r).  Of widened int8 values the eight lanes
  // that write at once hold chunks of one parity: two to a bank, but for the bit of c (128 values) or r (64) that goes into
  // the lowest.  (The conflicts cost no time that shows: 1000 queries over 30000 keys 787 us with and without them, 300
  // launches each.)
  // Rows of bfloat16 come straight to LDS and need none of it (a prompt of 128 values 642 us with it, 637 without).
  __device__ static __forceinline__ int at(int c, int low) { return kI8 ? c ^ c >> 3 ^ low : c + low; }
  __device__ static __forceinline__ int fk(int r) { return kChunks == 16 ? r & 15 : ((r >> 1) & 7) ^ (kI8 ? r & 1 : 0); }
  __device__ static __forceinline__ int fv(int r) { return kChunks == 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1) ^ (kI8 ? r & 1 : 0); }
};

template <int D, bool kI8>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) paged_attn_chunk_kernel(AttnArgs, Parts P, int most, int least_log2) {
  using T = ChunkTile<D, kI8>;
  using Value = std::conditional_t<kI8, int8_t, __bf16>;
  constexpr int kSteps = D / 16, kOut = D / 32, kElem = kI8 ? 1 : 2;
  constexpr int kGlobalChunks = D * kElem / 16;           // 16-byte pieces of a row in the cache
  constexpr int kRowsPerCopy = 64 / kGlobalChunks;        // rows that one access of a wave brings
  constexpr int kCopies = 16 / kRowsPerCopy;              // accesses for 16 rows
  __shared__ __attribute__((aligned(1024))) char s_kv[2][2][T::kBytes];  // [buffer][keys, values]
  __shared__ __attribute__((aligned(16))) float s_scale[2][2][kI8 ? 64 : 4];
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups go round the eight dies; neighbours in the list of items share keys, so a die takes consecutive workers.
  const int me = most % 8 ? blockIdx.x : (blockIdx.x & 7) * (most / 8) + (blockIdx.x >> 3);
  Schedule<T::kKeys> sched;
  int64_t u, u1;
  Item I;
  int at;
  if (!sched.start(args_anew(), me, most, least_log2, u, u1, I, at)) {
    if (threadIdx.x == 0) P.note[me] = int4{-1, 0, 0, 0};
    return;
  }
  // A lane's part of an access: row crow (+ kRowsPerCopy i) of the quarter, 16-byte piece cpiece.
  const int crow = lane / kGlobalChunks, cpiece = lane % kGlobalChunks;
  const uint32_t lds0 = lds_addr(s_kv);
  int buf = 0;
  bool noted = false;
  uint32_t kts, vts, kat[kCopies], vat[kCopies], page_mask;  // bytes from token to token, and where the lane's pieces come from
  float mul;
  {
    const AttnArgs& A = args_anew();
    kts = static_cast<uint32_t>(A.c.k_stride[2]) * kElem;
    vts = static_cast<uint32_t>(A.c.v_stride[2]) * kElem;
    page_mask = A.c.page_size - 1;
    // A scale of zero is queries of zero (times infinity a weight would be NaN).
    mul = A.scale == 0.0f ? 1.0f : fabsf(A.scale) * kLog2e;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int row = i * kRowsPerCopy + crow;  // (the permutations repeat after 16 rows)
      kat[i] = row * kts + 16 * (kI8 ? cpiece : cpiece ^ T::fk(row));
      vat[i] = row * vts + 16 * (kI8 ? cpiece : cpiece ^ T::fv(row));
    }
  }

  while (u < u1) {
    const int k0 = at, k1 = static_cast<int>(min(static_cast<int64_t>(I.units), k0 + (u1 - u)));
    // The page ids of this wave's quarter of 64 tiles, a lane each (-1: names no page), read together and waited for here
    // (one read for every tile would be waited for in every tile); and for each quarter which tiles' ids name none.
    int ids = 0, ids_from = 0;
    uint64_t none[4];
    bool named = false;  // a page of this worker's tiles is one of the cache's
    const auto read_ids = [&](int kt) {
      const AttnArgs& A = args_anew();
      const int32_t* trow = A.table + static_cast<int64_t>(I.r) * A.width;
      ids_from = kt;
      int all[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int key0 = 64 * (I.t0 + kt + lane) + 16 * x;
        all[x] = key0 < I.hi && key0 + 16 > I.lo ? trow[key0 >> A.page_shift] : -1;
      }
      wait_vmem_all();
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool bad = all[x] < 0 || all[x] >= A.c.pages;
        const int key0 = 64 * (I.t0 + kt + lane) + 16 * x;
        none[x] = __ballot(bad && key0 < I.hi && key0 + 16 > I.lo);
        named |= __any(!bad && kt + lane < k1);
        if (x == wave) ids = bad ? -1 : all[x];
      }
    };
    // Where the item's keys and values lie (kv head h of page 0), bytes from page to page, and of the scales.
    const char *kbase, *vbase, *ksbase, *vsbase;
    uint32_t kps, vps, sps;
    // The 16 rows of key tile kt that this wave brings: resources that end behind the last key that any query sees.
    // (Rows before the first are read as they are.)
    const auto quarter_of = [&](int kt, u32x4 (&Q)[4]) {
      const int key0 = 64 * (I.t0 + kt) + 16 * wave;
      const int id = __builtin_amdgcn_readlane(ids, kt - ids_from);
      const uint32_t page = max(id, 0), off = key0 & page_mask;
      const int n = id < 0 ? 0 : max(0, min(16, I.hi - key0));
      Q[0] = raw_rsrc(kbase + static_cast<uint64_t>(page) * kps + off * kts, n ? (n - 1) * kts + D * kElem : 0);
      Q[1] = raw_rsrc(vbase + static_cast<uint64_t>(page) * vps + off * vts, n ? (n - 1) * vts + D * kElem : 0);
      if constexpr (kI8) {
        Q[2] = raw_rsrc(ksbase + static_cast<uint64_t>(page) * sps + off * 4, 4 * n);
        Q[3] = raw_rsrc(vsbase + static_cast<uint64_t>(page) * sps + off * 4, 4 * n);
      }
    };
    // bfloat16: rows straight to LDS.
    const auto copy_tile = [&](int kt, int b) {
      u32x4 Q[4];
      quarter_of(kt, Q);
      const uint32_t dst = lds0 + b * 2 * T::kBytes + 16 * wave * T::kRow;
      copy16<false>(Q[0], kat, dst);
      copy16<false>(Q[1], vat, dst + T::kBytes);
    };
    // int8: rows to registers, and from there, widened, to LDS.
    u32x4 rk[kCopies], rv[kCopies];
    float rks = 0.0f, rvs = 0.0f;
    const auto load_tile = [&](int kt) {
      u32x4 Q[4];
      quarter_of(kt, Q);
      const auto rsrc = [](u32x4 r) { return make_rsrc(reinterpret_cast<const void*>(static_cast<uint64_t>(r[1]) << 32 | r[0]), r[2]); };
      const auto k = rsrc(Q[0]), v = rsrc(Q[1]);
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        rk[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k, kat[i], 0, 0));
        rv[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(v, vat[i], 0, 0));
      }
      rks = as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc(Q[2]), lane * 4, 0, 0));
      rvs = as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc(Q[3]), lane * 4, 0, 0));
    };
    // One of kPieces equal parts of the tile; the scales go with the first.
    constexpr int kPieces = 4 * kCopies;
    const auto store_piece = [&](int b, int piece) {
      const int i = piece / 4, x = piece / 2 % 2, row = 16 * wave + i * kRowsPerCopy + crow;
      if (piece % 2 == 0)
        *reinterpret_cast<bf16x8*>(s_kv[b][0] + row * T::kRow + 16 * (T::at(2 * cpiece, x) ^ T::fk(row))) = widen8(u32x2{rk[i][2 * x], rk[i][2 * x + 1]});
      else
        *reinterpret_cast<bf16x8*>(s_kv[b][1] + row * T::kRow + 16 * (T::at(2 * cpiece, x) ^ T::fv(row))) = widen8(u32x2{rv[i][2 * x], rv[i][2 * x + 1]});
      if (piece == 0 && lane < 16) {
        s_scale[b][0][16 * wave + lane] = rks;
        s_scale[b][1][16 * wave + lane] = rvs;
      }
    };
    const auto store_tile = [&](int b) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) store_piece(b, i);
    };

    const int row = 32 * wave + c;
    int rows, rlo, rhi;                   // of the item; the keys that the lane's row sees
    int any_lo, any_hi, all_lo, all_hi;  // that some of the wave's rows see, that all of them see
    bf16x8 q[kSteps];
    {
      const AttnArgs& A = args_anew();
      kbase = static_cast<const char*>(A.c.k) + kElem * I.h * A.c.k_stride[1];
      vbase = static_cast<const char*>(A.c.v) + kElem * I.h * A.c.v_stride[1];
      kps = static_cast<uint32_t>(kElem * A.c.k_stride[0]);
      vps = static_cast<uint32_t>(kElem * A.c.v_stride[0]);
      ksbase = reinterpret_cast<const char*>(A.c.k_scale + static_cast<int64_t>(I.h) * A.c.page_size);
      vsbase = reinterpret_cast<const char*>(A.c.v_scale + static_cast<int64_t>(I.h) * A.c.page_size);
      sps = 4u * A.c.kv_heads * A.c.page_size;
      // `buf` is not the last item's last tile's: every wave has left it (it passed that tile's barrier).
      read_ids(k0);
      if constexpr (kI8) {
        load_tile(k0);
        store_tile(buf);
        if (k0 + 1 < k1) load_tile(k0 + 1);
      } else {
        copy_tile(k0, buf);
      }
      rows = I.count * A.group;
      const int tok = static_cast<int>(row * A.group_inv >> 16), head = row - tok * A.group;
      const bool on = row < rows;
      const int64_t t = I.s.q0 + I.first + tok, hq = static_cast<int64_t>(I.h) * A.group + head;
      seen(A, I.s, I.first + tok, rlo, rhi);
      if (!on || rhi < rlo) rlo = rhi = 0;
      const uint32_t sign = A.scale < 0.0f ? 0x80008000u : 0u;  // a negative scale goes into the queries' signs
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        u32x4 w{0, 0, 0, 0};
        if (on && A.scale != 0.0f) w = *reinterpret_cast<const u32x4*>(A.q + t * A.qs[0] + hq * A.qs[1] + 16 * s + 8 * h);
        q[s] = __builtin_bit_cast(bf16x8, w ^ sign);
      }
      const int wfirst = static_cast<int>(32 * wave * A.group_inv >> 16);
      const int wlast = static_cast<int>((min(rows, 32 * wave + 32) - 1) * A.group_inv >> 16);
      seen(A, I.s, I.first + wfirst, any_lo, all_hi);
      seen(A, I.s, I.first + wlast, all_lo, any_hi);
      if (32 * wave >= rows) any_hi = 0;
    }

    if constexpr (!kI8) wait_vmem_all();  // the queries (and the first tile): no wait for them inside the loop
    f32x16 acc[kOut];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[o][i] = 0.0f;

    for (int kt = k0; kt < k1; ++kt, buf ^= 1) {
      const int key0 = 64 * (I.t0 + kt);
      if constexpr (!kI8) copies_left<0>();
      lds_reads_done();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const char* sk = s_kv[buf][0];
      const char* sv = s_kv[buf][1];
      if (kt + 2 - ids_from > 63) read_ids(kt);
      int bads = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) bads |= static_cast<int>(none[x] >> (kt - ids_from) & 1) << x;
      // Tiles that none of the wave's rows sees; of an int8 cache it still brings its part of the next tile, below.
      const bool blank = key0 >= any_hi || key0 + 64 <= any_lo;
      if constexpr (!kI8) {
        if (kt + 1 < k1) copy_tile(kt + 1, buf ^ 1);
        if (blank) continue;
      }
      const bool edge = key0 < all_lo || key0 + 64 > all_hi || bads;
      f32x16 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
      // Operands of two steps are read while those of the two before are multiplied: the compiler would read each one
      // just before its product and wait for it (a fence keeps it from that).
      const auto keys = [&](int st, bf16x8 (&a)[4]) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = 32 * (x & 1) + c;
          a[x] = *reinterpret_cast<const bf16x8*>(sk + r * T::kRow + 16 * (T::at(2 * (st + x / 2), h) ^ T::fk(r)));
        }
      };
      bf16x8 ka[2][4];
      keys(0, ka[0]);
      keys(2, ka[1]);
#pragma unroll
      for (int st = 0; st < kSteps; st += 2) {
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 (&a)[4] = ka[st / 2 % 2];
#pragma unroll
        for (int x = 0; x < 4; ++x) s[x & 1] = mfma32(a[x], q[st + x / 2], s[x & 1]);
        if (st + 4 < kSteps) keys(st + 4, a);
        // int8: the next tile is widened and stored between the products, which leave every other issue cycle free (after
        // the last tile a part of no tile, into a buffer that is filled anew).
        if constexpr (kI8) {
#pragma unroll
          for (int i = 0; i < 2 * kPieces / kSteps; ++i) store_piece(buf ^ 1, st / 2 * (2 * kPieces / kSteps) + i);
        }
      }
      if constexpr (kI8) {
        __builtin_amdgcn_sched_barrier(0);
        if (kt + 2 < k1) load_tile(kt + 2);
        if (blank) continue;
      }
      if constexpr (kI8) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(&s_scale[buf][0][32 * b + 8 * a + 4 * h]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[b][4 * a + i] *= w[i];
          }
      }
      // Whether the lane's row does not see its key i (of 32).
      const auto key_of = [&](int i) { return 32 * (i / 16) + 8 * (i / 4 % 4) + i % 4; };  // + 4 h + key0
      const int from = rlo - key0 - 4 * h;
      const uint32_t span = rhi - rlo;
      const auto unseen = [&](int i) { return static_cast<uint32_t>(key_of(i) - from) >= span; };
      if (edge) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (unseen(i)) s[i / 16][i % 16] = -INFINITY;
        if (bads) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (bads >> (i / 8) & 1) s[i / 16][i % 16] = -INFINITY;
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
      {
        const auto p = __builtin_amdgcn_permlane32_swap(as_uint(top), as_uint(top), false, false);
        top = fmaxf(as_float(p[0]), as_float(p[1])) * mul;
      }
      // The reference is raised only where a score passes it by more than 2^8: weights up to 2^8 lose nothing, and most
      // tiles then leave the sums as they are.
      if (__any(top > m + 8.0f)) {  // (m = -infinity: any score passes it)
        const float m1 = fmaxf(m, top), keep = m1 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= keep;
#pragma unroll
        for (int o = 0; o < kOut; ++o) acc[o] *= keep;
      }
      // Values of 32 of the head's values and 16 keys, transposed: the left operand.
      const auto values = [&](int o, int kb) {
        bf16x8 a;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int r = 16 * kb + 8 * x + 4 * h + (lane & 15) / 4;
          const int ch = T::at(4 * o, 2 * ((lane >> 4) & 1) + (lane & 3) / 2);
          const char* src = sv + r * T::kRow + 16 * (ch ^ T::fv(r)) + 8 * (lane & 1);
          const bf16x4 w = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)src));
#pragma unroll
          for (int i = 0; i < 4; ++i) a[4 * x + i] = w[i];
        }
        return a;
      };
      bf16x8 va[2][kOut];
#pragma unroll
      for (int o = 0; o < kOut; ++o) va[0][o] = values(o, 0);
      __builtin_amdgcn_sched_barrier(0);
      const float ref = m == -INFINITY ? 0.0f : m;
      bf16x8 p[4];
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      // Weights of 16 keys; those of the next 16 are formed between the products of these: a product takes a matrix core
      // 32 cycles, in 16 of which the vector unit can issue.
      const auto weigh = [&](int kb) {
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = __builtin_amdgcn_exp2f(fmaf(s[kb / 2][8 * (kb % 2) + i], mul, -ref));
          sum[i % 4] += w[i];
        }
        if constexpr (kI8) {
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(&s_scale[buf][1][16 * kb + 8 * a + 4 * h]);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * a + i] *= v[i];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) p[kb][i] = static_cast<__bf16>(w[i]);
      };
      weigh(0);
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        if (kb < 3) {
#pragma unroll
          for (int o = 0; o < kOut; ++o) va[(kb + 1) % 2][o] = values(o, kb + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int o = 0; o < kOut; ++o) acc[o] = mfma32(va[kb % 2][o], p[kb], acc[o]);
        if (kb < 3) {
          weigh(kb + 1);
          // A product, then a share of the vector instructions (left to the compiler's order: 1000 queries over 30000 int8
          // keys 814 us, so 808 us).
#pragma unroll
          for (int x = 0; x < kOut; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, 28 / kOut, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }

    const AttnArgs& A = args_anew();
    const bool whole = k0 == 0 && k1 == I.units, on = row < rows;
    const int tok = static_cast<int>(row * A.group_inv >> 16);
    const int64_t t = I.s.q0 + I.first + tok, hq = static_cast<int64_t>(I.h) * A.group + row - tok * A.group;
    const int slot = k0 > 0 ? kHead : kTail;
    {
      const auto p = __builtin_amdgcn_permlane32_swap(as_uint(l), as_uint(l), false, false);
      l = as_float(p[0]) + as_float(p[1]);
    }
    // The weights 2^(s mul - m) take the product s mul as it is, but m, one of these products, rounded: a factor on all of
    // them that the division by their sum takes out again, at most 2^(2^-5) up to |m| = 2^20.  Where m is huge it drives
    // them all to zero or infinity: beyond that bound rows are done again, with one rounding for both.
    bool odd = on && ((named && nothing_seen(A, I, tok, m, 64 * (I.t0 + k0), 64 * (I.t0 + k1))) || (m > -INFINITY && fabsf(m) > 0x1p20f));
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= !__builtin_isfinite(acc[o][i]);
    odd = __any(odd);
    if (odd) {
      rows_again<Value, D>(A, P, I, me, slot, whole, 64 * (I.t0 + k0), 64 * (I.t0 + k1), 32 * wave, min(rows, 32 * wave + 32));
    } else if (on && whole) {
      const bool none = m == -INFINITY && l == 0.0f;
      const float inv = none ? 0.0f : 1.0f / l;
      uint16_t* dst = A.out + t * A.os[0] + hq * A.os[1];
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          bf16x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = static_cast<__bf16>(none ? 0.0f : acc[o][4 * a + i] * inv);
          *reinterpret_cast<u32x2*>(dst + 32 * o + 8 * a + 4 * h) = __builtin_bit_cast(u32x2, w);
        }
      if (A.lse && h == 0) A.lse[t * A.q_heads + hq] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else if (on) {
      float* pacc = P.acc + ((static_cast<int64_t>(me) * 2 + slot) * P.rows + row) * D;
      float* pml = P.ml + ((static_cast<int64_t>(me) * 2 + slot) * P.rows + row) * 2;
#pragma unroll
      for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<f32x4*>(pacc + 32 * o + 8 * a + 4 * h) = f32x4{acc[o][4 * a], acc[o][4 * a + 1], acc[o][4 * a + 2], acc[o][4 * a + 3]};
      if (h == 0) {
        pml[0] = m;
        pml[1] = l;
      }
    }
    if (k1 < I.units) {
      noted = true;
      if (threadIdx.x == 0) P.note[me] = sched.note(I, u, k0, rows);
    }
    u += k1 - k0;
    at = 0;
    if (u < u1 && !sched.next(A, I)) break;
  }
  if (!noted && threadIdx.x == 0) P.note[me] = int4{-1, 0, 0, 0};
}

}  // namespace bitcos_attn
