// What the attention kernels share: the work's division over the workgroups, the cache's
// addresses, the parts of a split unit.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace basek {

// A unit is a tile of R packed rows of one sequence and key head: packed row r is the
// query head hk G + r % G of the sequence's new token r / G, so that the G query heads
// that share a key head go through the matrix instructions together.  Its cost is the
// number of blocks of BK keys its rows see (at least 1).  All units in the order
// (sequence, key head, tile) form one line of N blocks, and workgroup w of W takes the
// stretch [w per, (w + 1) per), whatever the lengths are: a unit that lies in several
// stretches is left in parts (the running maximum, the sum and the unnormalised output)
// that k_attn_join adds in their order.
struct AttnPart {
  int token, head, r0, n, slot, count, w, pad;   // count parts: slot, then 2 (w + 1), 2 (w + 2), ..
};

struct AttnArgs {
  HeadRows q, o;
  float *lse;
  KvCache c;
  KvBatch b;
  int rows, Hq, G, D, window;
  float scale;              // of the products, times log2 e
  int above, upto;          // sequences of more than `above` and at most `upto` packed rows
  int W;                    // workgroups
  bool whole;               // every unit costs 1 and is done by one workgroup
  float *part;
  AttnPart *rec;            // [W]: the unit that begins in workgroup w and ends in another
};

// One sequence: its first row, new tokens (all, and those taken), keys, packed rows
struct AttnSeq {
  int first, n, kv, packed;
  int pos0;                 // the first new token's position (may be below 0)
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int s) {
  AttnSeq q;
  const int begin = min(max(a.b.q_start[s], 0), a.rows);
  const int end = min(max(a.b.q_start[s + 1], begin), a.rows);
  const long long room = (long long)a.b.max_pages << a.c.shift;
  q.first = begin;
  q.kv = (int)min((long long)max(a.b.kv_len[s], 0), room);
  q.pos0 = q.kv - (end - begin);
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
  const int p0 = q.pos0 + r0 / a.G, p1 = q.pos0 + (r0 + n - 1) / a.G;
  k.hi = max(p1 + 1, 0);
  k.lo = a.window > 0 ? max(p0 - a.window + 1, 0) : 0;
  return k;
}

// a value that is the same in all lanes, known as such to the compiler
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uni(long long v) {
  return (long long)(((unsigned long long)(unsigned)uni((int)(v >> 32)) << 32) | (unsigned)uni((int)v));
}

template <int R, int BK>
struct AttnWork {
  const AttnArgs &a;
  long long at, end;        // of this workgroup's stretch, what is left
  long long per;
  int w;
  // where it stands: a sequence, its cost a head, the place inside it
  int s;
  AttnSeq q;
  int tiles;
  long long head_cost, rem;
  bool first;

  __device__ int tile_cost(const AttnSeq &sq, int j) const {
    if (a.whole) return 1;
    const KeyRange k = attn_keys(a, sq, j * R, min(R, sq.packed - j * R));
    const int c = (k.hi + BK - 1) / BK - k.lo / BK;
    return c > 1 ? c : 1;
  }
  __device__ long long cost_a_head(const AttnSeq &sq) const {
    const int t = (sq.packed + R - 1) / R;
    if (a.whole) return t;
    long long c = 0;
    for (int j = 0; j < t; ++j) c += tile_cost(sq, j);
    return c;
  }

  __device__ AttnWork(const AttnArgs &args, int w_) : a(args), w(w_), first(true) {
    const int lane = lane_id();
    long long c = 0, total = 0;
    for (int s0 = 0; s0 < a.b.n_seq; s0 += WAVE) {
      c = s0 + lane < a.b.n_seq ? cost_a_head(attn_seq(a, s0 + lane)) * a.c.Hk : 0;
      total += c;
    }
#pragma unroll
    for (int h = 1; h < WAVE; h *= 2) total += __shfl_xor(total, h, WAVE);
    total = uni(total);
    per = (total + a.W - 1) / a.W;
    if (per < 1) per = 1;
    at = w * per;
    end = at + per < total ? at + per : total;
    s = a.b.n_seq;
    rem = 0;
    if (at >= end) return;
    long long run = 0;
    for (int s0 = 0; s0 < a.b.n_seq; s0 += WAVE) {
      if (a.b.n_seq > WAVE) c = s0 + lane < a.b.n_seq ? cost_a_head(attn_seq(a, s0 + lane)) * a.c.Hk : 0;
      long long incl = c;
#pragma unroll
      for (int h = 1; h < WAVE; h *= 2) {
        const long long o = __shfl_up(incl, h, WAVE);
        if (lane >= h) incl += o;
      }
      const unsigned long long hit = __ballot(run + incl > at);
      if (hit) {
        const int l = __ffsll(hit) - 1;
        s = s0 + l;
        rem = at - run - __shfl(incl - c, l, WAVE);
        break;
      }
      run += __shfl(incl, WAVE - 1, WAVE);
    }
    s = uni(s);
    rem = uni(rem);
    enter();
  }
  __device__ void enter() {
    q = attn_seq(a, s);
    tiles = (q.packed + R - 1) / R;
    head_cost = cost_a_head(q);
  }

  // The next segment: blocks [k0, k1) of a unit whose rows are r0 .. r0 + n - 1 of the
  // sequence q and key head hk; `slot` is the part's place, -1 where the segment is all
  // of the unit
  struct Segment {
    int hk, r0, n, k0, k1, slot;
    KeyRange keys;
  };
  __device__ bool next(Segment &g, AttnPart &begun) {
    if (at >= end) return false;
    while (rem >= head_cost * a.c.Hk) {
      ++s;
      rem = 0;
      enter();
    }
    g.hk = (int)(rem / head_cost);
    int left = (int)(rem - g.hk * head_cost), j = 0, c;
    while (left >= (c = tile_cost(q, j))) {
      left -= c;
      ++j;
    }
    g.r0 = j * R;
    g.n = min(R, q.packed - g.r0);
    g.keys = attn_keys(a, q, g.r0, g.n);
    const int base = a.whole ? 0 : g.keys.lo / BK;
    const int take = (int)min((long long)(c - left), end - at);
    g.k0 = base + left;
    g.k1 = g.k0 + take;
    g.slot = -1;
    if (a.whole) {
      g.k0 = g.keys.lo / BK;
      g.k1 = (g.keys.hi + BK - 1) / BK;
    } else if (take < c) {
      g.slot = 2 * w + (first ? 0 : 1);
      if (left == 0) {   // the unit begins here and goes on
        const int last = (int)((at + c - 1) / per);
        begun = {q.first, g.hk * a.G, g.r0, g.n, g.slot, last - w + 1, w, 0};
      }
    }
    first = false;
    at += take;
    rem += take;
    return true;
  }
};

// A part: R rows of DP floats, then R maxima (of the products times scale log2 e) and R sums
template <int R, int DP>
__host__ __device__ constexpr size_t attn_part_floats() { return (size_t)R * (DP + 2); }

__device__ __forceinline__ int attn_page(const AttnArgs &a, int s, int key) {
  const int page = a.b.table[s * a.b.table_ld + (key >> a.c.shift)];
  // a page that is not in the cache is read as its first: in bounds
  return (unsigned)page < (unsigned)a.c.n_pages ? page : 0;
}

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.44269504088896341f;

}  // namespace basek
