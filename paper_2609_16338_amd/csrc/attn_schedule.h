// How attention is dealt out: equal shares of key tiles, whatever the lengths.
//
// A row tile is the queries of up to `tt` consecutive tokens of a request
// times the query heads of one kv head; with the tiles of kTile keys that any
// of its queries sees it makes an item, and its key tiles are the item's units
// (one unit where no key is seen: the empty rows are written too).  All items
// stand in one list -- request by request, kv head by kv head, row tile by row
// tile -- and worker x of w takes units [x U / w, (x + 1) U / w).  An item that
// ends up with several workers leaves unnormalised parts that a second launch
// joins in key order.  So one long context among short ones, a prompt among
// single tokens, or a single sequence fill the GPU alike; the lengths are read
// on the device, and the host needs to know no more than a sensible w.
//
// Every wave finds its place by itself: a lane per request counts units, a
// scan gives the total and the request, and a second scan over the row tiles
// of that request the item.
#pragma once

#include "attn_common.h"

namespace bitcos_attn {

// Unnormalised parts of an item: per worker one for an item begun before its
// range (kHead) and one for an item that goes on after it (kTail), each
// `rows` x dim sums over values and per row the maximum (base 2) and the sum
// of weights; and per worker a note of an item that goes on after its range.
struct Parts {
  float* acc;    // [workers][2][rows][dim]
  float* ml;     // [workers][2][rows][2]
  int4* note;    // [workers]: what the worker's parts but for a last one belong to: first token (-1: none), kv head,
                 // rows | first worker << 8, last worker
  int32_t rows;  // most rows of a row tile
};
enum { kHead = 0, kTail = 1 };

struct Item {
  int r, h, rt;
  Span s;
  int tiles;       // row tiles of the request
  int t0, units;   // first key tile, key tiles (at least 1)
  int lo, hi;      // keys that any of its queries sees
  int first, count;  // tokens of the request
};

template <int kTile>
struct Schedule {
  int64_t total = 0;  // units of all items (below 2^40: the host sees to it, for requests that share no token)
  int workers = 0;    // that share them

  static __device__ __forceinline__ int tiles_of(const AttnArgs& A, int n) {
    if (A.tt == 1) return n;
    return static_cast<int>(__umul64hi(static_cast<uint64_t>(n + A.tt - 1), A.tt_inv));
  }

  static __device__ __forceinline__ int tile_units(const AttnArgs& A, const Span& S, int rt, int& t0, int& klo, int& khi) {
    const int first = rt * A.tt, last = min(S.n, first + A.tt) - 1;
    int lo, hi, x;
    seen(A, S, first, lo, x);
    seen(A, S, last, x, hi);
    klo = lo;
    khi = max(hi, 0);
    t0 = lo / kTile;
    return max(1, (khi + kTile - 1) / kTile - t0);
  }

  // Units of one kv head's items of each lane's request: a loop over its row
  // tiles, or where there are many a loop over requests with a row tile a lane.
  static __device__ __forceinline__ int64_t head_units(const AttnArgs& A, const Span& S, int lane) {
    const int tiles = tiles_of(A, S.n);
    int64_t sum = 0;
    int a, b, c;
    if (tiles <= 4)
      for (int rt = 0; rt < tiles; ++rt) sum += tile_units(A, S, rt, a, b, c);
    uint64_t many = __ballot(tiles > 4);
    while (many) {
      const int src = __builtin_ctzll(many);
      many &= many - 1;
      Span T;
      T.n = __builtin_amdgcn_readlane(S.n, src);
      T.kv = __builtin_amdgcn_readlane(S.kv, src);
      T.q0 = 0;
      const int n = tiles_of(A, T.n);
      int64_t part = 0;
      for (int rt = lane; rt < n; rt += 64) part += tile_units(A, T, rt, a, b, c);
#pragma unroll
      for (int o = 32; o >= 1; o /= 2) part += __shfl_xor(part, o, 64);
      if (lane == src) sum = part;
    }
    return sum;
  }

  static __device__ __forceinline__ Span lane_span(const AttnArgs& A, int r) {
    Span S{0, 0, 0};
    if (r < A.requests) S = span_of(A, r);
    return S;
  }

  static __device__ __forceinline__ int64_t incl_scan(int64_t v, int lane) {
    if (!__any(v >= (1 << 25))) return wave_incl_scan(static_cast<int>(v));  // the sum fits 32 bits
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(v, d, 64);
      if (lane >= d) v += o;
    }
    return v;
  }
  // a / b for 0 <= a < 2^52, b > 0, rounded down.  The double quotient cannot round up to a whole number that the exact
  // one stays below: the two would differ by at least 1 / b, more than half a unit in the last place of a / b.
  static __device__ __forceinline__ int64_t divided(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);  // a third of the time
    return static_cast<int64_t>(static_cast<double>(a) / static_cast<double>(b));
  }
  static __device__ __forceinline__ int64_t lane_value(int64_t v, int src) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), src);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), src);
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  }

  static __device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(v));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32));
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  }

  static __device__ __forceinline__ void fill(const AttnArgs& A, Item& I) {
    I.units = tile_units(A, I.s, I.rt, I.t0, I.lo, I.hi);
    I.first = I.rt * A.tt;
    I.count = min(A.tt, I.s.n - I.first);
  }

  // The item of unit u0 of worker x's range [u0, u1), and u0's place in it;
  // false where the range is empty.  `most`: workers of the launch; a worker
  // has at least 2^least_log2 units, so that a short list is not cut too fine.
  __device__ __forceinline__ bool start(const AttnArgs& A, int x, int most, int least_log2, int64_t& u0, int64_t& u1, Item& I, int& at) {
    const int lane = threadIdx.x & 63;
    // Twice over the requests, 64 at a time: for the total, then to the request that holds u0.
    Span S;
    int64_t per_head, incl, base = 0;
    int r0 = 0;
    bool place = false;
    while (true) {
      S = lane_span(A, r0 + lane);
      per_head = head_units(A, S, lane);
      incl = incl_scan(per_head * A.c.kv_heads, lane);
      const int64_t here = lane_value(incl, 63);
      if (!place) {
        total += here;
        if (total >> 40) return false;  // cu_q that does not ascend: nothing is done, rather than numbers that wrap
        if (r0 + 64 < A.requests) {
          r0 += 64;
          continue;
        }
        const int64_t share = (total + (1 << least_log2) - 1) >> least_log2;
        workers = static_cast<int>(share < most ? share : most);
        if (x >= workers) return false;
        u0 = uniform(divided(x * total, workers));
        u1 = uniform(divided((x + 1) * total, workers));
        place = true;
        if (r0 == 0) break;  // one round held them all
        r0 = 0;
        continue;
      }
      if (u0 < base + here) break;
      base += here;
      r0 += 64;
      if (r0 >= A.requests) return false;  // (lengths that changed under way: no endless search)
    }
    const int src = __builtin_ctzll(__ballot(base + incl > u0));
    const int64_t heads = lane_value(per_head, src);
    int64_t left = u0 - base - (lane_value(incl, src) - heads * A.c.kv_heads);
    I.r = r0 + src;
    I.s.q0 = __builtin_amdgcn_readlane(S.q0, src);
    I.s.n = __builtin_amdgcn_readlane(S.n, src);
    I.s.kv = __builtin_amdgcn_readlane(S.kv, src);
    I.tiles = tiles_of(A, I.s.n);
    I.h = static_cast<int>(uniform(divided(left, heads)));
    left -= I.h * heads;
    I.rt = 0;
    at = static_cast<int>(left);
    for (int rt0 = 0; I.tiles > 1 && rt0 < I.tiles; rt0 += 64) {
      int a, b, c;
      const int rt = rt0 + lane;
      const int64_t run = incl_scan(rt < I.tiles ? tile_units(A, I.s, rt, a, b, c) : 0, lane);
      const uint64_t past = __ballot(run > left);
      if (past) {
        const int w = __builtin_ctzll(past);
        I.rt = rt0 + w;
        at = static_cast<int>(left - (w ? lane_value(run, w - 1) : 0));
        break;
      }
      left -= lane_value(run, 63);
    }
    fill(A, I);
    return true;
  }

  // The next item of the list; false where there is none.
  static __device__ __forceinline__ bool next(const AttnArgs& A, Item& I) {
    if (++I.rt == I.tiles) {
      I.rt = 0;
      if (++I.h == A.c.kv_heads) {
        I.h = 0;
        do {
          if (++I.r >= A.requests) return false;
          const Span S = span_of(A, I.r);
          I.s.q0 = __builtin_amdgcn_readfirstlane(S.q0);
          I.s.n = __builtin_amdgcn_readfirstlane(S.n);
          I.s.kv = __builtin_amdgcn_readfirstlane(S.kv);
        } while (I.s.n == 0);
        I.tiles = tiles_of(A, I.s.n);
      }
    }
    fill(A, I);
    return true;
  }

  // The note of a worker at unit u, place k0 of item I, whose part of it ends before the item does.
  __device__ __forceinline__ int4 note(const Item& I, int64_t u, int k0, int rows) const {
    return int4{I.s.q0 + I.first, I.h, rows | worker_of(u - k0) << 8, worker_of(u - k0 + I.units - 1)};
  }

  // The worker that has unit u.
  __device__ __forceinline__ int worker_of(int64_t u) const {
    return static_cast<int>(uniform(divided((u + 1) * workers - 1, total)));
  }
};

}  // namespace bitcos_attn
