// What the attention kernels share: the work's division over the workgroups, the cache's
// addresses, the parts of a split unit.
#pragma once

#include "common.hpp"
#include "internal.hpp"
#include "seq.hpp"

namespace basek {

// A unit is a tile of R packed rows of one sequence and key head: packed row r is the
// query head hk G + r % G of the sequence's new token r / G, so that the G query heads
// that share a key head go through the matrix instructions together.  Its cost is the
// number of blocks of BK keys its rows see (at least 1) and a pad in front of them, for
// what a change of units costs.  All units in the order
// (sequence, key head, tile) form one line of N blocks, and workgroup w of W takes the
// stretch [w per, (w + 1) per), whatever the lengths are: a unit that lies in several
// stretches is left in parts (the running maximum, the sum and the unnormalised output)
// that k_attn_join adds in their order.  A workgroup's parts lie at 2 w (its first
// segment) and 2 w + 1.
struct AttnPart {   // the unit that goes on behind a workgroup's stretch
  int token, head, r0, n;
  int slot, count, w, pad;   // count parts from workgroup w on: slot, 2 (w + 1), 2 (w + 2), ..
};

// x / by for 0 <= x < 2^31, by a product: by's m = floor(2^(31 + shift) / by) + 1 with
// 2^shift >= by is too large by less than 2^-31 of itself (the host makes it)
struct Divisor {
  uint32_t m;
  int shift;
};
inline Divisor divisor(uint32_t by) {
  Divisor d{0, 0};
  while ((1ull << d.shift) < by) ++d.shift;
  d.m = (uint32_t)((1ull << (31 + d.shift)) / by + 1);
  return d;
}
__device__ __forceinline__ int over(int x, Divisor d) {
  return (int)(((uint64_t)(uint32_t)x * d.m) >> (31 + d.shift));
}
// x / y for 0 <= x < 2^31, 0 < y, with a quotient below 2^20
__device__ __forceinline__ int quotient(int x, int y) {
  int q = (int)((float)x * __builtin_amdgcn_rcpf((float)y));
  int r = x - q * y;
  if (r < 0) { --q; r += y; }
  if (r >= y) ++q;
  return q;
}

struct AttnArgs {
  HeadRows q, o;
  float *lse;
  KvCache c;
  KvBatch b;
  int rows, Hq, G, D, window;
  Divisor by_G, by_W;
  float scale;              // of the products, times log2 e
  int above, upto;          // sequences of more than `above` and at most `upto` packed rows
  int W;                    // workgroups
  int coarse;               // a cost is of 2^coarse blocks
  uint32_t limit;           // the line is no longer
  int pad;                  // what a unit costs besides its blocks
  bool whole;               // every unit costs 1 and is done by one workgroup
  float *part;
  AttnPart *rec;            // [W]
};

// One sequence: its first row, keys, new tokens taken, packed rows, and the first new
// token's position (may be below 0)
struct AttnSeq {
  int first, kv, n, packed, pos0;
};
// from its rows [begin, end) and keys, taken within their bounds
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int begin, int end, int kv) {
  AttnSeq q;
  q.first = begin;
  q.kv = kv;
  q.pos0 = kv - (end - begin);
  q.n = min(end - begin, a.b.max_q);
  q.packed = q.n * a.G;
  if (q.packed <= a.above || q.packed > a.upto) q.packed = 0;
  return q;
}

// Keys [lo, hi) that the rows r0 .. r0 + n - 1 see between them
struct KeyRange {
  int lo, hi;
};
__device__ __forceinline__ KeyRange attn_keys(const AttnArgs &a, const AttnSeq &q, int r0, int n) {
  KeyRange k;
  const int p0 = q.pos0 + over(r0, a.by_G), p1 = q.pos0 + over(r0 + n - 1, a.by_G);
  k.hi = max(p1 + 1, 0);
  k.lo = a.window > 0 ? max(max(p0, 0) - a.window + 1, 0) : 0;
  return k;
}

// a value that is the same in all lanes, known as such to the compiler
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The same value, of which the compiler knows nothing: what follows from it is not computed
// in front of a loop (the masks and addresses of a unit's rows would hold 80 registers
// through the loop over the keys)
__device__ __forceinline__ int here(int v) {   // uniform
  asm volatile("" : "+s"(v));
  return v;
}
__device__ __forceinline__ int lane_here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The value of lane ^ 16 or lane ^ 32 beside the lane's own, in one or the other order (an
// exchange of rows of 16 lanes, or of the halves, between two copies: no way through LDS)
template <int H>
__device__ __forceinline__ void both_lanes(float v, float &x, float &y) {
  static_assert(H == 16 || H == 32, "lane distance");
  const unsigned u = __float_as_uint(v);
  const auto r = H == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                         : __builtin_amdgcn_permlane32_swap(u, u, false, false);
  x = __uint_as_float(r[0]);
  y = __uint_as_float(r[1]);
}
template <int H>
__device__ __forceinline__ float max_lane(float v) {
  float x, y;
  both_lanes<H>(v, x, y);
  return fmaxf(x, y);
}
template <int H>
__device__ __forceinline__ float add_lane(float v) {
  float x, y;
  both_lanes<H>(v, x, y);
  return x + y;
}

__device__ __forceinline__ int wave_sum(int v) {
  const int lane = lane_here(lane_id());
#pragma unroll
  for (int h = 1; h < WAVE; h *= 2) v += __builtin_amdgcn_ds_bpermute(4 * (lane ^ h), v);
  return v;
}
// inclusive, and 2^32 - 1 where it is more
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
  const int lane = lane_here(lane_id());
#pragma unroll
  for (int h = 1; h < WAVE; h *= 2) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane - h), (int)v);
    if (lane >= h) v = __builtin_elementwise_add_sat(v, o);
  }
  return v;
}

// The walk of a workgroup over its stretch of the line (costs in units of 2^a.coarse
// blocks, so that the line of `rows` rows is shorter than 2^30; starts on the device that
// fall and rise again can make it longer than rows can, and then nothing is done).  Lane l
// holds sequence s0 + l.
template <int R, int BK>
struct AttnWork {
  const AttnArgs &a;
  int w, per, at, end;      // the stretch's rest
  int s0, begin, stop, kv, cost;   // of the lane's sequence; cost: a head's
  int s, hk, j, left;       // where it stands: sequence, key head, tile, place in the tile
  int tiles;
  int q0, q1, len;          // of the lane's sequence of the next 64, as they are in memory
  AttnSeq q;
  bool first;
  static constexpr int LANE_TILES = 16;

  __device__ int tile_cost(const AttnSeq &sq, int j) const {
    if (a.whole) return 1;
    const KeyRange k = attn_keys(a, sq, j * R, min(R, sq.packed - j * R));
    const int c = ((k.hi + BK - 1) / BK - k.lo / BK + (1 << a.coarse) - 1) >> a.coarse;
    return a.pad + (c > 1 ? c : 1);
  }
  __device__ AttnSeq lane_seq(int l) const {
    return attn_seq(a, __builtin_amdgcn_readlane(begin, l), __builtin_amdgcn_readlane(stop, l),
                    __builtin_amdgcn_readlane(kv, l));
  }
  __device__ void fetch(int from) {   // the sequences from .. from + 63, for load
    const int i = min(from + lane_id(), a.b.n_seq - 1);
    q0 = a.b.q_start[i];
    q1 = a.b.q_start[i + 1];
    len = a.b.kv_len[i];
  }
  // (the next 64 are fetched while these are taken: in a batch of 256 a workgroup would wait
  // eight times for memory before its first key)
  __device__ void load(int from) {
    s0 = from;
    const int lane = lane_id();
    const SeqRows rows = seq_rows(q0, q1, len, a.rows, a.b.max_pages << a.c.shift);
    begin = rows.begin;
    stop = rows.stop;
    kv = rows.kv;
    if (from + lane >= a.b.n_seq) stop = begin;
    if (a.b.n_seq > WAVE) fetch(from + WAVE < a.b.n_seq ? from + WAVE : 0);
    const AttnSeq sq = attn_seq(a, begin, stop, kv);
    const int t = (sq.packed + R - 1) / R;
    if (a.whole) {
      cost = t;
      return;
    }
    // a lane the tiles of its sequence, or where they are many, all lanes those of one
    cost = 0;
    for (int i = 0; i < t && t <= LANE_TILES; ++i) cost += tile_cost(sq, i);
    unsigned long long more = __ballot(t > LANE_TILES);
    while (more) {
      const int l = __ffsll(more) - 1;
      more &= more - 1;
      const AttnSeq one = lane_seq(l);
      const int n = (one.packed + R - 1) / R;
      int c = 0;
      for (int t0 = lane; t0 < n; t0 += WAVE) c += tile_cost(one, t0);
      c = wave_sum(c);
      if (lane == l) cost = c;
    }
  }

  __device__ AttnWork(const AttnArgs &args, int w_) : a(args), w(w_), first(true) {
    // the line's length, then the place of the stretch's begin in it: the second pass needs
    // no loads where one chunk of 64 holds all sequences
    uint32_t total = 0, incl = 0;
    int run = 0;
    bool placed = false;
    at = end = 0;
    fetch(0);
    for (int from = 0;;) {
      if (!placed || a.b.n_seq > WAVE) {
        load(from);
        incl = wave_prefix(cost * a.c.Hk);
      }
      const uint32_t sum = (uint32_t)__builtin_amdgcn_readlane((int)incl, WAVE - 1);
      if (!placed) {
        total = __builtin_elementwise_add_sat(total, sum);
        from += WAVE;
        if (from < a.b.n_seq) continue;
        if (total > a.limit) return;
        per = max(over((int)total + a.W - 1, a.by_W), 1);
        at = min(w * (long long)per, (long long)total);
        end = min(at + per, (int)total);
        if (at >= end) return;
        placed = true;
        from = 0;
        if (a.b.n_seq > WAVE) continue;
      }
      const unsigned long long hit = __ballot(run + (int)incl > at);
      if (hit) {
        const int l = __ffsll(hit) - 1, head = __builtin_amdgcn_readlane(cost, l);
        left = at - run - __builtin_amdgcn_readlane((int)incl, l) + head * a.c.Hk;
        const int rest = left;
        enter(from + l);
        hk = quotient(rest, head);
        left = rest - hk * head;
        break;
      }
      run += sum;
      from += WAVE;
    }
    // the tile with that place, 64 tiles at a time
    for (int j0 = 0; tiles > 1; j0 += WAVE) {
      const int c = j0 + lane_id() < tiles ? tile_cost(q, j0 + lane_id()) : 0, upto = (int)wave_prefix(c);
      const unsigned long long in = __ballot(upto > left);
      if (in) {
        const int m = __ffsll(in) - 1;
        j = j0 + m;
        left -= __builtin_amdgcn_readlane(upto - c, m);
        break;
      }
      left -= __builtin_amdgcn_readlane(upto, WAVE - 1);
    }
  }
  __device__ void enter(int i) {
    s = i;
    q = lane_seq(i - s0);
    tiles = (q.packed + R - 1) / R;
    hk = j = left = 0;
  }

  // The next segment: blocks [k0, k1) of a unit whose rows are r0 .. r0 + n - 1 of the
  // sequence q and key head hk; `slot` is the part's place, -1 where the segment is all
  // of the unit
  struct Segment {
    int s, hk, r0, n, k0, k1, slot;
    AttnSeq q;
    KeyRange keys;
  };
  __device__ bool next(Segment &g, AttnPart &begun) {
    if (at >= end) return false;
    if (j == tiles) {
      j = 0;
      ++hk;
    }
    if (hk == a.c.Hk) {   // on to the next sequence that has work
      unsigned long long more = __ballot(cost > 0) & (s - s0 == WAVE - 1 ? 0ull : ~0ull << (s - s0 + 1));
      while (!more) {
        load(s0 + WAVE);
        more = __ballot(cost > 0);
      }
      enter(s0 + __ffsll(more) - 1);
    }
    const int c = tile_cost(q, j);
    if (left < a.pad) {   // the unit's blocks begin behind its pad, if in this stretch at all
      const int skip = min(a.pad - left, end - at);
      at += skip;
      left += skip;
      if (at >= end) return false;
    }
    g.s = s;
    g.q = q;
    g.hk = hk;
    g.r0 = j * R;
    g.n = min(R, q.packed - g.r0);
    g.keys = attn_keys(a, q, g.r0, g.n);
    const int take = min(c - left, end - at), b0 = g.keys.lo / BK, b1 = (g.keys.hi + BK - 1) / BK;
    g.k0 = a.whole ? b0 : b0 + ((left - a.pad) << a.coarse);
    g.k1 = take == c - left ? b1 : b0 + ((left - a.pad + take) << a.coarse);
    g.slot = take < c - a.pad ? 2 * w + (first ? 0 : 1) : -1;
    if (left + take < c) {   // the unit goes on in the next workgroup
      const int from = at - left, w0 = quotient(from + a.pad, per);
      begun = {q.first, hk * a.G, g.r0, g.n, 2 * w0 + (from <= w0 * per ? 0 : 1),
               quotient(from + c - 1, per) - w0 + 1, w0, 0};
    }
    first = false;
    at += take;
    left = 0;
    ++j;
    return true;
  }
};

// A part: pieces of 64 lanes times four adjoining elements as the accumulators lie, ROWS rows'
// (32 in k_attn_many, 16 in k_attn_few) after another's, R DP floats in all; then R maxima (of
// the products times scale log2 e) and R sums.  Piece q of lane l holds row ROWS (q / per) + l
// % ROWS, per = ROWS DP / 256, and four elements from attn_at on.
template <typename T, int ROWS, int DP>
__device__ __forceinline__ int attn_at(int q, int lane) {
  const int in = q % (ROWS * DP / 256);
  if (sizeof(T) == 4) return 64 * (in / 4) + 16 * (lane / 16) + 4 * (in % 4);
  return ROWS == 32 ? 8 * in + 4 * (lane / 32) : 16 * in + 4 * (lane / 16);
}
template <int R, int DP>
__host__ __device__ constexpr size_t attn_part_floats() { return (size_t)R * (DP + 2); }

__device__ __forceinline__ int attn_page(const AttnArgs &a, int s, int key) {
  const int page = a.b.table[s * a.b.table_ld + (key >> a.c.shift)];
  // a page that is not in the cache is read as its first: in bounds
  return (unsigned)page < (unsigned)a.c.n_pages ? page : 0;
}

typedef __attribute__((address_space(3))) void *lds_p;

// 16 bytes per lane from global memory to LDS, lane l's at lds + 16 l (lds uniform).  The
// compiler's builtin makes every transposed read wait for all such loads, those of the
// steps ahead among them; here the reader waits for its own (wait_vm).  No register is
// written; a wait of the compiler's for a load of its own is only the longer for these.
__device__ __forceinline__ uint32_t lds_addr(const void *p) {
  return (uint32_t)(uintptr_t)(lds_p)p;
}
__device__ __forceinline__ void glb_to_lds(const char *p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
// the same from a uniform address and a lane's offset.  The address may come out of a
// vector register right in front of this (lane_at, or a spilled scalar's reload), and a
// vector-memory instruction may read such a scalar only five wait states after it was
// written; the hardware does not wait by itself, nor does the compiler look in here.  The
// move and s_nop 3 are those five.
__device__ __forceinline__ void glb_to_lds(const char *base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
// the address in lane l's registers
__device__ __forceinline__ const char *lane_at(uint32_t lo, uint32_t hi, int l) {
  return (const char *)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32) |
                        (uint32_t)__builtin_amdgcn_readlane((int)lo, l));
}

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.44269504088896341f;

// What a row's sum comes to: 0 and -infinity where it has no key, NaN where the sum is NaN
__device__ __forceinline__ float inverse(float sum) {
  return sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
}
__device__ __forceinline__ float log_sum(float top, float sum) {
  return sum > 0.0f ? (top + __log2f(sum)) * LN2 : (sum == 0.0f ? -INFINITY : sum);
}

}  // namespace basek
