// Attention of each sequence's new tokens over its paged cache:
//   o = sum_j e^(c q.k_j - m) v_j / sum_j e^(c q.k_j - m)    over the keys j that the
// token sees (its own position and those before it, of a window if there is one), in one
// pass over the keys with the running maximum m and sum.
//
// The products are made transposed, S^T = K Q^T and O^T = V^T P^T: a lane's accumulators
// then belong to one packed row (query head and token), so m and the sum are values of
// the lane, and S^T's registers, rounded, are the operand P^T of the second product as
// they lie: its keys are taken in the order in which the first product left them.
//
// k_attn_few: tiles of 16 or 32 packed rows, the wavefronts on blocks of keys of their own,
// joined through LDS at the unit's end.  16-bit rows come asynchronously to a ring in
// LDS (wavefront's own: no barrier in the loop), where 16-byte pieces are permuted so that
// neither product's operand reads meet in a bank; V's operand is read transposed.  Bound by
// the cache's reads: 256 sequences of 1000 keys and 16 heads of 128 (2.1 GB) 367 us, 5.7
// TB/s; one of 131071 keys and 4 heads (268 MB) 54 us; short calls by the chain of loads to
// the first key: 517 keys 8 us.  Two wavefronts a workgroup, as many workgroups as the
// LDS of a CU holds rings of two steps: what is in flight is what counts.
#include "attn.hpp"
#include "ffn.hpp"

namespace basek {

namespace {

// 16 bytes of zeros: what a lane reads in the place of a key or element that is not there
__device__ __attribute__((aligned(16))) uint32_t g_zero[4];

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 *lds_b4;

// The addresses of K's and V's rows from a token on (16-bit), one token a lane: made for many
// steps at once, and read lane by lane (in scalar registers their 64-bit products took 1100
// of a block's 6000 cycles in k_attn_many).  A page that is not in the cache is read as its
// first: in bounds.
struct RowAt {
  uint32_t klo, khi, vlo, vhi;
};
__device__ __forceinline__ RowAt row_at(const AttnArgs &a, int s, int hk, int key) {
  const long long page = attn_page(a, s, key), slot = key & ((1 << a.c.shift) - 1);
  const uint64_t k = (uint64_t)a.c.k + 2 * (page * a.c.k_page + slot * a.c.k_slot + hk * a.c.k_head);
  const uint64_t v = (uint64_t)a.c.v + 2 * (page * a.c.v_page + slot * a.c.v_slot + hk * a.c.v_head);
  return {(uint32_t)k, (uint32_t)(k >> 32), (uint32_t)v, (uint32_t)(v >> 32)};
}
// Four 16-bit elements a lane, transposed in groups of 16 lanes: lane 4 r + c gives the
// address of elements 4 c .. + 3 of row r, and lane i gets element i of the rows 0 .. 3
__device__ __forceinline__ bf16x4 read_tr(const char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b4)(lds_p)p);
}

struct __attribute__((packed, aligned(2))) Any16H { u32x4 v; };
struct __attribute__((packed, aligned(4))) Any16F { f32x4 v; };
struct __attribute__((packed, aligned(2))) Any8H { u32x2 v; };

__device__ __forceinline__ void put4(uint16_t *p, f32x4 v) {
  u32x2 q;
  q[0] = (uint32_t)f32_to_bf16_any(v[0]) | ((uint32_t)f32_to_bf16_any(v[1]) << 16);
  q[1] = (uint32_t)f32_to_bf16_any(v[2]) | ((uint32_t)f32_to_bf16_any(v[3]) << 16);
  reinterpret_cast<Any8H *>(p)->v = q;
}
__device__ __forceinline__ void put4(float *p, f32x4 v) { reinterpret_cast<Any16F *>(p)->v = v; }

// m's rise that is left to the products' exponents: P stays below 2^LAG, and the
// accumulators are rescaled only when the maximum has risen by more
constexpr float LAG = 8.0f;

// Workgroups a CU of k_attn_few.  16-bit: what its LDS holds.  fp32: with 16 rows of 128
// elements two have registers (10 sequences of 21974 keys 273 us, one workgroup 361); with 32
// rows short calls lose by the parts of twice the workgroups (64 tokens of 2048 keys 35.7 us
// against 29.9, 300 of 1000 36.2 against 30.8; 13 of 21974, 28 heads on 7, 602 against 672)
constexpr int few_occ(bool bf, int dp, int nr) {
  return bf ? (dp == 64 ? 4 : dp == 128 ? 2 : 1) : dp * nr <= 128 ? 2 : 1;
}
template <typename T, int DP_, int NR_>
struct FewShape {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int DP = DP_, NR = NR_, R = 16 * NR;
  static constexpr int TK = BF ? 32 : 16;                  // keys of a wavefront's step
  static constexpr int WAVES = BF ? 2 : 4, THREADS = WAVES * WAVE, BK = WAVES * TK;
  static constexpr int CH = DP / 8;                        // 16-byte pieces of a 16-bit row
  static constexpr int ROWB = DP * 2, STAGE = 2 * TK * ROWB, RING = 2, LOADS = CH;
  static constexpr int STATE = DP * 64 + 512;              // 16 rows of a wavefront's state
  static constexpr int AREA = (WAVES - 1) * STATE, LDS = (BF ? WAVES * RING * STAGE : 0) + AREA;
  static constexpr int OCC = few_occ(BF, DP, NR);
  static constexpr int WPE = OCC * WAVES >= 4 ? OCC * WAVES / 4 : 1;
  static_assert(OCC * LDS <= 160 * 1024, "LDS of a CU");
};

// pieces' places in a row of the ring: K's row r at piece ^ few_k(r), V's at piece ^ few_v(r)
template <int CH> __device__ __forceinline__ int few_k(int r) { return CH == 8 ? (r >> 1) & 7 : r & 15; }
template <int CH> __device__ __forceinline__ int few_v(int r) { return CH == 8 ? 2 * ((r >> 1) & 3) : 2 * (r & 7); }

template <typename T, int DP, int NR>
__global__ __launch_bounds__((FewShape<T, DP, NR>::THREADS), (FewShape<T, DP, NR>::WPE))
void k_attn_few(AttnArgs a) {
  using M = FewShape<T, DP, NR>;
  constexpr bool BF = M::BF;
  constexpr int R = M::R, TK = M::TK;
  constexpr int DT = DP / 16;                     // accumulator tiles
  constexpr int QS = BF ? DP / 32 : DP / 16;      // operand pieces of 16 bytes
  using Work = AttnWork<R, M::BK>;
  __shared__ __attribute__((aligned(256))) char lds[M::LDS];
  const int wave = wave_id_u(), lane = lane_id(), n = lane % 16, g = lane / 16;
  const char *zero = reinterpret_cast<const char *>(g_zero);
  char *const area = lds + M::LDS - M::AREA;
  // the lane's places in the loads of a step (piece j of 64 16-byte pieces)
  uint32_t ko[BF ? M::CH / 2 : 1], vo[BF ? M::CH / 2 : 1];
  uint32_t kin = 0, vin = 0;   // bit j: the piece is one of the head's D elements
  if constexpr (BF) {
#pragma unroll
    for (int j = 0; j < M::CH / 2; ++j) {
      const int row = (lane + WAVE * j) / M::CH, piece = (lane + WAVE * j) % M::CH;
      ko[j] = 2 * ((row & 15) * (uint32_t)a.c.k_slot + 8 * (piece ^ few_k<M::CH>(row)));
      vo[j] = 2 * ((row & 15) * (uint32_t)a.c.v_slot + 8 * (piece ^ few_v<M::CH>(row)));
      if (8 * (piece ^ few_k<M::CH>(row)) < a.D) kin |= 1u << j;
      if (8 * (piece ^ few_v<M::CH>(row)) < a.D) vin |= 1u << j;
    }
  }
  char *const ring = lds + wave * M::RING * M::STAGE;
  const uint32_t ring_at = lds_addr(ring);
  // heads shorter than DP: K's places past D, which no load of a whole step writes, are zeros
  // from here on (V's hold anything: they are sums of their own, which nobody stores)
  if (BF && a.D < DP) {
#pragma unroll 1
    for (int j = 0; j < M::CH / 2 * M::RING; ++j)
      *reinterpret_cast<u32x4 *>(ring + j / (M::CH / 2) * M::STAGE + j % (M::CH / 2) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // A segment as the wavefront has it: its steps i0 .. i1 - 1 (keys key0(i) .. + TK - 1),
  // the next one to request, and the addresses of 32 steps, two a step (16 keys lie in one
  // page): lane e has those of step from + e / 2
  struct Seg {
    typename Work::Segment g;
    int i0, i1, ask, from;
    RowAt at;
  };
  auto key0 = [&](int i) { return i * M::BK + wave * TK; };
  auto fetch_rows = [&](Seg &z, int i) {
    z.from = i;
    const int key = key0(i + lane / 2) + 16 * (lane & 1);
    z.at = row_at(a, z.g.s, z.g.hk, max(min(key, (z.g.keys.hi - 1) & ~15), 0));
  };
  auto steps = [&](Seg &z) {
    z.i0 = max(z.g.k0, (z.g.keys.lo - wave * TK) / M::BK);
    z.i1 = min(z.g.k1, (z.g.keys.hi - wave * TK + M::BK - 1) / M::BK);
    // (a quotient rounds to zero, where the bound above or below holds)
    while (z.i0 < z.i1 && key0(z.i0) + TK <= z.g.keys.lo) ++z.i0;
    z.i1 = max(z.i1, z.i0);
    z.ask = z.i0;
  };
  auto queries = [&](const typename Work::Segment &sg, u32x4 (&qv)[NR][QS]) {
    const int D = here(a.D);
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const int r = 16 * c + n, pr = sg.r0 + min(r, sg.n - 1), tok = over(pr, a.by_G);
      const T *p = (const T *)a.q.p + (long long)(sg.q.first + tok) * a.q.row +
                   (long long)(sg.hk * a.G + pr - tok * a.G) * a.q.head;
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        const int d = BF ? 32 * s + 8 * g : 16 * s + 4 * g;
        const T *at = p + min(d, D - (BF ? 8 : 4));
        if constexpr (BF) qv[c][s] = reinterpret_cast<const Any16H *>(at)->v;
        else qv[c][s] = __builtin_bit_cast(u32x4, reinterpret_cast<const Any16F *>(at)->v);
      }
    }
  };
  auto take_queries = [&](u32x4 (&to)[NR][QS], const u32x4 (&raw)[NR][QS]) {
    const int D = here(a.D);
#pragma unroll
    for (int c = 0; c < NR; ++c)
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        const uint32_t keep = (BF ? 32 * s + 8 * lane_here(g) : 16 * s + 4 * lane_here(g)) < D ? ~0u : 0u;
        to[c][s] = raw[c][s] & keep;
      }
  };
  // The segment's next step into the stage given.  Rows of it that no token sees are brought
  // too: 16 keys lie in one page, and in place of a page that is not there another is read.
  auto issue = [&](Seg &z, int stage) {
    const int i = z.ask++;
    if (i - z.from >= 32) fetch_rows(z, i);
    const uint32_t st = ring_at + stage * M::STAGE;
    const char *kb[2], *vb[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      kb[h] = lane_at(z.at.klo, z.at.khi, 2 * (i - z.from) + h);
      vb[h] = lane_at(z.at.vlo, z.at.vhi, 2 * (i - z.from) + h);
    }
    if (a.D == DP) {
#pragma unroll
      for (int j = 0; j < M::CH / 2; ++j) {
        const int h = WAVE * j / M::CH / 16;
        glb_to_lds(kb[h], ko[j], st + j * 1024);
        glb_to_lds(vb[h], vo[j], st + TK * M::ROWB + j * 1024);
      }
    } else {   // (some lanes of each load have a piece: all are issued, as wait_vm counts)
#pragma unroll
      for (int j = 0; j < M::CH / 2; ++j) {
        const int h = WAVE * j / M::CH / 16;
        if (kin >> j & 1) glb_to_lds(kb[h], ko[j], st + j * 1024);
        if (vin >> j & 1) glb_to_lds(vb[h], vo[j], st + TK * M::ROWB + j * 1024);
      }
    }
  };

  AttnPart begun{};
  Work work(a, blockIdx.x);
  // z: the segment at hand, ahead: the next one, whose queries and addresses are loaded (16-bit) and
  // whose first steps are requested behind z's last, so that between segments the memory is
  // not left waiting; src: the one whose steps are being requested
  Seg z, ahead, src;
  u32x4 qv[NR][QS], qn[NR][BF ? QS : 1];
  int asked = 0, used = 0;   // steps requested and used, of all segments: the ring's places
  bool have = false, more = true, early = false;   // early: src is ahead
  while (true) {
    if (more) {
      more = work.next(ahead.g, begun);
      if (more) {
        steps(ahead);
        if constexpr (BF) {
          queries(ahead.g, qn);
          fetch_rows(ahead, ahead.i0);
          // waited for here, where what is in flight besides has been for long: the compiler's
          // wait at their first use would be for the steps requested since, too
#pragma unroll
          for (int c = 0; c < NR; ++c)
#pragma unroll
            for (int s = 0; s < QS; ++s) asm volatile("" ::"v"(qn[c][s]));
          asm volatile("" ::"v"(ahead.at.klo));
        }
      }
    }
    if (!have) {
      if (!more) break;
      have = true;
      z = src = ahead;
      if constexpr (BF) take_queries(qv, qn);
      continue;
    }
    const typename Work::Segment &sg = z.g;
    if constexpr (!BF) {   // (nothing is requested ahead here, and there are no registers to spare)
      queries(sg, qv);
      take_queries(qv, qv);
    }
    const int lo = sg.keys.lo, hi = sg.keys.hi, nr = NR > 1 && sg.n > 16 ? 2 : 1, D = here(a.D);
    int pos[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const int r = 16 * c + n;
      pos[c] = r < sg.n ? max(sg.q.pos0 + over(sg.r0 + min(r, sg.n - 1), a.by_G), -1) : -1;
    }
    const int pmin = sg.q.pos0 + over(sg.r0, a.by_G), pmax = sg.q.pos0 + over(sg.r0 + sg.n - 1, a.by_G);
    f32x4 acc[NR][DT];
    float m[NR], l[NR];
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.0f;
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[c][t] = f32x4{0, 0, 0, 0};
    }

    // p (for the second product) from the products of a step, and m, l, acc's scale
    auto soften = [&](int c, int k0, float (&x)[TK / 4]) {
      const bool cut = k0 + TK - 1 > pmin || (a.window > 0 && k0 <= pmax - a.window) || c * 16 + 16 > sg.n;
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < TK / 4; ++e) x[e] = x[e] * a.scale;
      if (cut) {
#pragma unroll
        for (int e = 0; e < TK / 4; ++e) {
          const int key = k0 + 16 * (e / 4) + 4 * g + e % 4;
          const bool seen = key <= pos[c] && (a.window == 0 || key > pos[c] - a.window);
          x[e] = seen ? x[e] : -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < TK / 4; ++e) top = fmaxf(top, x[e]);
      top = max_lane<32>(max_lane<16>(top));
      if (__any(top > m[c] + LAG)) {
        const float to = fmaxf(m[c], top), f = m[c] == to ? 1.0f : __builtin_amdgcn_exp2f(m[c] - to);
        m[c] = to;
        l[c] *= f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[c][t][e] *= f;
      }
      const float mm = m[c] == -INFINITY ? 0.0f : m[c];
#pragma unroll
      for (int e = 0; e < TK / 4; ++e) {
        x[e] = __builtin_amdgcn_exp2f(x[e] - mm);
        l[c] += x[e];
      }
    };

    for (int i = z.i0; i < z.i1; ++i) {
      const int k0 = key0(i);
      if constexpr (BF) {
        while (asked - used < M::RING) {
          if (src.ask == src.i1 && !early && more) {
            src = ahead;
            early = true;
          }
          if (src.ask == src.i1) break;
          issue(src, asked++ & 1);
        }
        if (asked - used > 1) wait_vm<M::LOADS>();
        else wait_vm<0>();
        char *st = ring + (used++ & 1) * M::STAGE, *sv = st + TK * M::ROWB;
        // V's rows that no token sees may hold anything: zeros (K's are masked as products)
        if (k0 < lo || k0 + TK > hi) {
#pragma unroll
          for (int j = 0; j < M::CH / 2; ++j) {
            const int key = k0 + (lane + WAVE * j) / M::CH;
            if (key < lo || key >= hi) *reinterpret_cast<u32x4 *>(sv + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
          }
          asm volatile("" ::: "memory");
        }
        f32x4 s[NR][2];
#pragma unroll
        for (int c = 0; c < NR; ++c) s[c][0] = s[c][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int q = 0; q < QS; ++q) {
            const int row = 16 * b + n;
            const bf16x8 kv = *reinterpret_cast<const bf16x8 *>(
                st + row * M::ROWB + (((4 * q + g) ^ few_k<M::CH>(row)) * 16));
            s[0][b] = mfma16(kv, __builtin_bit_cast(bf16x8, qv[0][q]), s[0][b]);
            if (nr > 1) s[NR - 1][b] = mfma16(kv, __builtin_bit_cast(bf16x8, qv[NR - 1][q]), s[NR - 1][b]);
          }
        // p as a bf16 and the bf16 of what that leaves: the second product is not what
        // bounds the kernel (within 2% of the time), and the output's error stays its own
        // rounding's (1.35 times that with one)
        bf16x8 p[NR], pl[NR];
#pragma unroll
        for (int c = 0; c < NR; ++c) {
          if (c < nr) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[c][e / 4][e % 4];
            soften(c, k0, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              p[c][e] = (__bf16)x[e];
              pl[c][e] = (__bf16)(x[e] - (float)p[c][e]);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const int row = 4 * g + n / 4, piece = 2 * t + (n & 3) / 2;
          const char *at = sv + row * M::ROWB + ((piece ^ few_v<M::CH>(row)) * 16) + (n & 1) * 8;
          const bf16x4 v0 = read_tr(at), v1 = read_tr(at + 16 * M::ROWB);
          const bf16x8 vv = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          acc[0][t] = mfma16(vv, p[0], acc[0][t]);
          acc[0][t] = mfma16(vv, pl[0], acc[0][t]);
          if (nr > 1) {
            acc[NR - 1][t] = mfma16(vv, p[NR - 1], acc[NR - 1][t]);
            acc[NR - 1][t] = mfma16(vv, pl[NR - 1], acc[NR - 1][t]);
          }
        }
        // this stage's reads are done before its next rows are requested
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      } else {
        const long long page = attn_page(a, sg.s, k0), slot = k0 & ((1 << a.c.shift) - 1);
        const float *kb = (const float *)a.c.k + page * a.c.k_page + slot * a.c.k_slot + sg.hk * a.c.k_head;
        const float *vb = (const float *)a.c.v + page * a.c.v_page + slot * a.c.v_slot + sg.hk * a.c.v_head;
        const float *zf = reinterpret_cast<const float *>(zero);
        f32x4 kv[QS];
        const bool kin = k0 + n >= lo && k0 + n < hi;
#pragma unroll
        for (int q = 0; q < QS; ++q) {
          const int d = 16 * q + 4 * g;
          kv[q] = *reinterpret_cast<const f32x4 *>(kin && d < D ? kb + n * a.c.k_slot + d : zf);
        }
        // (Which elements the tiles have is free: a lane's of four tiles adjoin, one load for
        // four.  64 sequences of 1000 keys, heads of 256: 240 us with a load each, 195.)
        f32x4 vv[4][DT / 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = k0 + 4 * g + e;
          const bool vin = key >= lo && key < hi;
#pragma unroll
          for (int j = 0; j < DT / 4; ++j)
            vv[e][j] = *reinterpret_cast<const f32x4 *>(
                vin && 64 * j + 4 * n < D ? vb + (4 * g + e) * a.c.v_slot + 64 * j + 4 * n : zf);
        }
        __builtin_amdgcn_sched_barrier(0);   // (left to itself the compiler moves them behind the first product)
#pragma unroll
        for (int c = 0; c < NR; ++c) {
          if (c >= nr) continue;
          f32x4 s = {0, 0, 0, 0};
#pragma unroll
          for (int q = 0; q < QS; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[q][e], __uint_as_float(qv[c][q][e]), s, 0, 0, 0);
          float x[4] = {s[0], s[1], s[2], s[3]};
          soften(c, k0, x);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < DT; ++t)
              acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[e][t / 4][t % 4], x[e], acc[c][t], 0, 0, 0);
        }
      }
    }

    // four adjoining elements of the lane's row: 16-bit a tile's, fp32 one of each of four tiles
    auto piece = [&](int c, int t) {
      if constexpr (BF) return acc[c][t];
      const int j = t / 4 * 4, e = t % 4;
      return f32x4{acc[c][j][e], acc[c][j + 1][e], acc[c][j + 2][e], acc[c][j + 3][e]};
    };
    // the wavefronts' states, added to the first one's in their order, 16 rows at a time
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      if (c >= nr) continue;
      l[c] = add_lane<32>(add_lane<16>(l[c]));
      lds_barrier();   // the area is free
      if (wave > 0) {
        char *to = area + (wave - 1) * M::STATE;
#pragma unroll
        for (int t = 0; t < DT; ++t) reinterpret_cast<f32x4 *>(to)[t * WAVE + lane] = acc[c][t];
        reinterpret_cast<float *>(to + DP * 64)[lane] = lane < 32 ? m[c] : l[c];   // (the same 16 twice)
      }
      lds_barrier();
      if (wave > 0) continue;
      float top = m[c];
#pragma unroll
      for (int v = 1; v < M::WAVES; ++v)
        top = fmaxf(top, reinterpret_cast<const float *>(area + (v - 1) * M::STATE + DP * 64)[n]);
      const float mm = top == -INFINITY ? 0.0f : top, f0 = __builtin_amdgcn_exp2f(m[c] - mm);
      float sum = l[c] * f0;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][t][e] *= f0;
#pragma unroll
      for (int v = 1; v < M::WAVES; ++v) {
        const char *of = area + (v - 1) * M::STATE;
        const float f = __builtin_amdgcn_exp2f(reinterpret_cast<const float *>(of + DP * 64)[n] - mm);
        sum = __builtin_fmaf(f, reinterpret_cast<const float *>(of + DP * 64)[32 + n], sum);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const f32x4 x = reinterpret_cast<const f32x4 *>(of)[t * WAVE + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[c][t][e] = __builtin_fmaf(f, x[e], acc[c][t][e]);
        }
      }
      const int r = 16 * c + n;
      if (r >= sg.n) continue;
      if (sg.slot >= 0) {
        float *part = a.part + sg.slot * attn_part_floats<R, DP>();
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4 *>(part + ((c * DT + t) * WAVE + lane) * 4) = piece(c, t);
        if (g == 0) {
          part[R * DP + r] = top;
          part[R * DP + R + r] = sum;
        }
      } else {
        const int pr = sg.r0 + r, tok = over(pr, a.by_G), head = sg.hk * a.G + pr - tok * a.G;
        const long long row = sg.q.first + tok;
        const float inv = inverse(sum);
        T *out = (T *)a.o.p + row * a.o.row + head * a.o.head;
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const int at = attn_at<T, 16, DP>(t, lane);
          if (at < D) put4(out + at, piece(c, t) * inv);
        }
        if (a.lse && g == 0) a.lse[row * a.Hq + head] = log_sum(top, sum);
      }
    }
    if (!more) break;
    z = ahead;
    if (!early) src = ahead;
    early = false;
    if constexpr (BF) take_queries(qv, qn);
  }
  if (!a.whole && threadIdx.x == 0) a.rec[blockIdx.x] = begun;
}

// ------------------------------------------------------------- chunks --
// k_attn_many: tiles of 32 packed rows a wavefront on 32x32x16 products, the workgroup's
// wavefronts on the same block of BK keys, whose rows they bring to a ring in LDS together.
// The products and the softmax between them take a SIMD about as long as each other, so
// its two wavefronts take turns: in phase 2 t the first half of the workgroup makes the
// products of block t (S = K Q^T) and of block t - 1 (O += V^T P^T), and the second half
// the softmax of block t - 1; in phase 2 t + 1 the other way round.
// 2048 new tokens of 8191, 32 heads of 128 on 4 key heads (240 GFLOP): the call 237 us, 1017
// TFLOP/s, the join's 15 us among them; of 3600 cycles a block 1330 products, 1160 softmax,
// 400 requests, the rest barriers and waits, at a clock of 2.0 GHz under this load, half of
// whose cycles the matrix pipe works.  More rows a wavefront have no registers, fewer share
// a block's keys among fewer rows.
template <int DP_>
struct ManyShape {
  static constexpr int DP = DP_, WAVES = DP == 256 ? 4 : 8, THREADS = WAVES * WAVE, R = 32 * WAVES;
  static constexpr int BK = DP == 256 ? 32 : 64, CH = DP / 8, ROWB = DP * 2, RING = 4;
  static constexpr int HALF = BK * ROWB, STAGE = 2 * HALF, LDS = RING * STAGE;
  static constexpr int PI = HALF / 1024 / WAVES;   // loads of K, and of V, a wavefront and block
  static constexpr int WPE = DP == 256 ? 1 : 2;
  static_assert(PI * WAVES * 1024 == HALF && WAVE / CH <= 16, "a load's rows lie in one page");
};
template <int CH> __device__ __forceinline__ int many_k(int r) { return CH == 8 ? (r >> 1) & 7 : r & 15; }
template <int CH> __device__ __forceinline__ int many_v(int r) { return CH == 8 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); }

typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// N products, each operand read from LDS AHEAD products before it (left to itself the
// compiler reads each in front of its product and waits for it: twice the time)
template <int N, int AHEAD, typename Read, typename Mul>
__device__ __forceinline__ void fed(Read read, Mul mul) {
  bf16x8 v[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) v[i] = read(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    mul(i, v[i % AHEAD]);
    if (i + AHEAD < N) v[i % AHEAD] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int DP>
__global__ __launch_bounds__((ManyShape<DP>::THREADS), (ManyShape<DP>::WPE))
void k_attn_many(AttnArgs a) {
  using M = ManyShape<DP>;
  constexpr int R = M::R, BK = M::BK, CH = M::CH, QS = DP / 16, DT = DP / 32, KB = BK / 32;
  __shared__ __attribute__((aligned(256))) char lds[M::LDS];
  const uint32_t ring_at = lds_addr(lds);
  const int wave = wave_id_u(), lane = lane_id(), n = lane % 32, h = lane / 32;
  const int w = a.W % N_XCD ? blockIdx.x : blockIdx.x % N_XCD * (a.W / N_XCD) + blockIdx.x / N_XCD;
  const char *zero = reinterpret_cast<const char *>(g_zero);
  // (one wavefront a SIMD has nobody to take turns with)
  const int half = M::WPE > 1 ? wave / (M::WAVES / 2) : 0;
  auto row0 = [&](int j) { return (wave + M::WAVES * j) * WAVE / CH; };   // of load j
  uint32_t ko[M::PI], vo[M::PI], kin = 0, vin = 0;                        // the lane's places in it, and which there are
#pragma unroll
  for (int j = 0; j < M::PI; ++j) {
    const int row = row0(j) + lane / CH;
    ko[j] = 2 * (lane / CH * (uint32_t)a.c.k_slot + 8 * (lane % CH ^ many_k<CH>(row)));
    vo[j] = 2 * (lane / CH * (uint32_t)a.c.v_slot + 8 * (lane % CH ^ many_v<CH>(row)));
    if (8 * (lane % CH ^ many_k<CH>(row)) < a.D) kin |= 1u << j;
    if (8 * (lane % CH ^ many_v<CH>(row)) < a.D) vin |= 1u << j;
  }
  // as in k_attn_few: K's places past D are zeros, V's anything
  if (a.D < DP) {
#pragma unroll 1
    for (int j = 0; j < M::PI * M::RING; ++j)
      *reinterpret_cast<u32x4 *>(lds + j / M::PI * M::STAGE + (j % M::PI * M::WAVES + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    lds_barrier();
  }
  const float scale = a.scale != 0.0f ? fabsf(a.scale) : 1.0f;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
  AttnPart begun{};
  AttnWork<R, BK> work(a, w);
  typename AttnWork<R, BK>::Segment sg;
  while (work.next(sg, begun)) {
    const int D = here(a.D);
    const int lo = sg.keys.lo, hi = sg.keys.hi;
    const int r = 32 * wave + n, pr = sg.r0 + min(r, sg.n - 1), tok = over(pr, a.by_G);
    const bool mine = 32 * wave < sg.n;
    const int pos = r < sg.n ? max(sg.q.pos0 + tok, -1) : -1;
    // positions of the wavefront's first and last row
    const int wlast = min(32 * wave + 31, sg.n - 1);
    const int pmin = sg.q.pos0 + over(sg.r0 + 32 * wave, a.by_G), pmax = sg.q.pos0 + over(sg.r0 + max(wlast, 0), a.by_G);
    u32x4 qv[QS];
    {
      const uint16_t *p = (const uint16_t *)a.q.p + (long long)(sg.q.first + tok) * a.q.row +
                          (long long)(sg.hk * a.G + pr - tok * a.G) * a.q.head;
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        const int d = 16 * s + 8 * lane_here(h);
        qv[s] = reinterpret_cast<const Any16H *>(p + min(d, D - 8))->v;
      }
    }
    f32x16 acc[DT];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][e] = 0.0f;

    // the addresses of 64 / PI blocks at a time: lane e has that of load e % PI of block
    // from + e / PI
    int from = sg.k0;
    RowAt rows{};
    auto fetch_rows = [&](int i) {
      from = i;
      const int key = (i + lane / M::PI) * BK + (wave + M::WAVES * (lane % M::PI)) * WAVE / CH;
      const int most = (hi - 1) / (WAVE / CH) * (WAVE / CH);
      rows = row_at(a, sg.s, sg.hk, min(key, most));
    };
    // blocks whose keys are all there
    const int full0 = (lo + BK - 1) / BK, full1 = hi / BK;
    auto issue = [&](int i) {
      if (__builtin_expect(i - from >= WAVE / M::PI, 0)) fetch_rows(i);
      const uint32_t st = ring_at + (i & (M::RING - 1)) * M::STAGE;
      const uint32_t to = st + row0(0) * M::ROWB;
      const char *kb[M::PI], *vb[M::PI];
#pragma unroll
      for (int j = 0; j < M::PI; ++j) {
        kb[j] = lane_at(rows.klo, rows.khi, M::PI * (i - from) + j);
        vb[j] = lane_at(rows.vlo, rows.vhi, M::PI * (i - from) + j);
      }
      if (__builtin_expect(i >= full0 && i < full1, 1)) {
        if (__builtin_expect(a.D == DP, 1)) {
#pragma unroll
          for (int j = 0; j < M::PI; ++j) {
            glb_to_lds(kb[j], ko[j], to + j * M::WAVES * 1024);
            glb_to_lds(vb[j], vo[j], to + j * M::WAVES * 1024 + M::HALF);
          }
        } else {
#pragma unroll
          for (int j = 0; j < M::PI; ++j) {
            if (kin >> j & 1) glb_to_lds(kb[j], ko[j], to + j * M::WAVES * 1024);
            if (vin >> j & 1) glb_to_lds(vb[j], vo[j], to + j * M::WAVES * 1024 + M::HALF);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < M::PI; ++j) {
          const int row = row0(j) + lane / CH, ck = lane % CH ^ many_k<CH>(row), cv = lane % CH ^ many_v<CH>(row);
          const bool in = i * BK + row >= lo && i * BK + row < hi;
          glb_to_lds(in && 8 * ck < a.D ? kb[j] + ko[j] : zero, to + j * M::WAVES * 1024);
          glb_to_lds(in && 8 * cv < a.D ? vb[j] + vo[j] : zero, to + j * M::WAVES * 1024 + M::HALF);
        }
      }
    };
    const int blocks = hi > 0 ? sg.k1 - sg.k0 : 0;
    if (blocks > 0) fetch_rows(sg.k0);
    // a negative scale is taken over by the queries' signs, 0 by queries of 0: the scaled
    // maximum is then the maximum scaled
#pragma unroll
    for (int s = 0; s < QS; ++s) {
      const uint32_t keep = a.scale != 0.0f && 16 * s + 8 * lane_here(h) < D ? ~0u : 0u;
      qv[s] = (qv[s] ^ flip) & keep;
    }
    if (blocks > 0) issue(sg.k0);
    if (blocks > 1) issue(sg.k0 + 1);
    if (blocks > 1) wait_vm<2 * M::PI>();
    else wait_vm<0>();
    lds_barrier();
    // blocks ta .. tb - 1: those that some row of the wavefront sees
    const int ta = a.window > 0 ? max(0, max(max(pmin, 0) - a.window + 1, 0) / BK - sg.k0) : 0;
    const int tb = mine ? min(blocks, (max(pmax, -1) + BK) / BK - sg.k0) : 0;
    auto seen_block = [&](int t) { return t >= ta && t < tb; };
    // the stage of block t + 1 is there (all wavefronts': each waits for its own loads)
    auto wait_next = [&](int t) {
      if (t + 2 < blocks) wait_vm<2 * M::PI>();
      else wait_vm<0>();
    };
    f32x16 s[KB];
    bf16x8 p[2 * KB];
    // operands of the products of block t: V^T of the keys 16 ks .., elements 32 d ..; K of
    // the keys 32 b .., elements 16 q ..  (many_v(row) is that of row + 8)
    const int vrow = 4 * h + (lane % 16) / 4;
    auto read_v = [&](int t, int i) {
      const char *sv = lds + ((sg.k0 + t) & (M::RING - 1)) * M::STAGE + M::HALF;
      const int ks = i / DT, piece = 4 * (i % DT) + (lane / 16 & 1) * 2 + (lane & 3) / 2;
      const char *at = sv + (16 * ks + vrow) * M::ROWB + ((piece ^ many_v<CH>(vrow)) * 16) + (lane & 1) * 8;
      const bf16x4 v0 = read_tr(at), v1 = read_tr(at + 8 * M::ROWB);
      return bf16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
    };
    auto read_k = [&](int t, int i) {
      const char *sk = lds + ((sg.k0 + t) & (M::RING - 1)) * M::STAGE;
      const int row = 32 * (i % KB) + n;
      return *reinterpret_cast<const bf16x8 *>(sk + row * M::ROWB + (((2 * (i / KB) + h) ^ many_k<CH>(row)) * 16));
    };
    auto mul_v = [&](int i, bf16x8 v) { acc[i % DT] = mfma32(v, p[i / DT], acc[i % DT]); };
    auto mul_k = [&](int i, bf16x8 v) {
      if (i < KB)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[i][e] = 0.0f;
      s[i % KB] = mfma32(v, __builtin_bit_cast(bf16x8, qv[i / KB]), s[i % KB]);
    };
    constexpr int NV = 2 * KB * DT, NK = QS * KB;
    // the second half runs one phase behind; each requests rows in its softmax's phase: those
    // of the block after next, whose stage's last readers have passed
    if (half) {
      if (blocks > 2) issue(sg.k0 + 2);
      lds_barrier();
    }
    for (int t = 0; t <= blocks; ++t) {
      const int late = here(half);   // (one loop for both halves, not one each)
      const bool old = seen_block(t - 1), now = seen_block(t);
      __builtin_amdgcn_s_setprio(1);
      if (old) fed<NV, 4>([&](int i) { return read_v(t - 1, i); }, mul_v);
      if (now) fed<NK, 4>([&](int i) { return read_k(t, i); }, mul_k);
      __builtin_amdgcn_s_setprio(0);
      if (late) wait_next(t);
      lds_barrier();
      if (t + 2 + late < blocks) issue(sg.k0 + t + 2 + late);
      if (now) {
        const int k0 = (sg.k0 + t) * BK;
        if (k0 + BK - 1 > pmin || (a.window > 0 && k0 <= pmax - a.window)) {
          // (key <= pos and > pos - window, the block's and the lane's part on one side)
          const int last = pos - k0 - 4 * h, first = a.window > 0 ? last - a.window : -0x40000000;
#pragma unroll
          for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int key = 32 * b + 8 * (e / 4) + e % 4;
              s[b][e] = key <= last && key > first ? s[b][e] : -INFINITY;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, s[b][e]);
        top = max_lane<32>(top) * scale;
        if (__any(top > m + LAG)) {
          const float to = fmaxf(m, top), f = m == to ? 1.0f : __builtin_amdgcn_exp2f(m - to);
          m = to;
          l *= f;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] *= f;
        }
        // p as one bf16 for the second product (not for the sums): the products bound this
        // kernel, and the rest as a second part makes the chunk above 321 us of 237 and a
        // mixed batch 51 of 47, for an error of 0.0017 in place of 0.0023
        const float mm = m == -INFINITY ? 0.0f : m;
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], scale, -mm));
            sums[e % 4] += x;
            p[2 * b + e / 8][e % 8] = (__bf16)x;
          }
        l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
      }
      if (!late) wait_next(t);
      lds_barrier();
    }
    if (!half) lds_barrier();
    l = add_lane<32>(l);
    const int d0 = lane_here(4 * h);   // the lane's first element
    if (r < sg.n) {
      if (sg.slot >= 0) {
        float *part = a.part + sg.slot * attn_part_floats<R, DP>();
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<f32x4 *>(part + (((wave * DT + t) * 4 + e / 4) * WAVE + lane) * 4) =
                f32x4{acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]};
        if (h == 0) {
          part[R * DP + r] = m;
          part[R * DP + R + r] = l;
        }
      } else {
        const int head = sg.hk * a.G + pr - tok * a.G;
        const long long row = sg.q.first + tok;
        const float inv = inverse(l);
        uint16_t *out = (uint16_t *)a.o.p + row * a.o.row + head * a.o.head;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            if (32 * t + 2 * e + d0 < D)
              put4(out + 32 * t + 2 * e + d0,
                   f32x4{acc[t][e] * inv, acc[t][e + 1] * inv, acc[t][e + 2] * inv, acc[t][e + 3] * inv});
        if (a.lse && h == 0) a.lse[row * a.Hq + head] = log_sum(m, l);
      }
    }
  }
  if (threadIdx.x == 0) a.rec[w] = begun;
}

// The parts of the units that lie in several workgroups' stretches, added in their order.
// Workgroup b takes its share of the unit that goes on behind stretch b: a unit of count
// parts has count - 1 workgroups.
template <typename T, int ROWS, int DP>
__device__ __forceinline__ void join_store(const AttnArgs &a, const AttnPart &p, int r, int q, float top,
                                           float sum, f32x4 o) {
  if (r >= p.n) return;
  const int pr = p.r0 + r, tok = over(pr, a.by_G), head = p.head + pr - tok * a.G, at = attn_at<T, ROWS, DP>(q, lane_id());
  const long long row = p.token + tok;
  const float inv = inverse(sum);
  if (at < a.D) put4((T *)a.o.p + row * a.o.row + head * a.o.head + at, o * inv);
  if (a.lse && at == 0) a.lse[row * a.Hq + head] = log_sum(top, sum);
}
// Sums of parts k0, k0 + step, .. (NB at a time, their loads together) of the pieces q0 ..
// q0 + PB - 1, which are of the same rows; r: the lane's
template <int R, int DP, int PB, int NB>
__device__ __forceinline__ void join_sum(const AttnArgs &a, const AttnPart &p, int r, int q0, int k0, int step,
                                         float &top, float &sum, f32x4 (&o)[PB]) {
  constexpr size_t F = attn_part_floats<R, DP>();
  // (a lane whose row is not there reads the last row's: nothing more from memory)
  constexpr int ROWS = R > 32 ? 32 : 16;
  const int past = max(r - (p.n - 1), 0), lane = lane_id() - past;
  r -= past;
  top = -INFINITY;
  sum = 0.0f;
#pragma unroll
  for (int b = 0; b < PB; ++b) o[b] = f32x4{0, 0, 0, 0};
  for (; k0 < p.count; k0 += NB * step) {
    float m[NB], l[NB];
    f32x4 x[NB][PB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int k = min(k0 + j * step, p.count - 1);
      const float *part = a.part + (k == 0 ? p.slot : 2 * (p.w + k)) * F;
      m[j] = part[R * DP + r];
      l[j] = part[R * DP + R + r];
#pragma unroll
      for (int b = 0; b < PB; ++b) x[j][b] = *reinterpret_cast<const f32x4 *>(part + ((q0 + b) * WAVE + lane) * 4);
    }
    float to = top;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (k0 + j * step >= p.count) m[j] = -INFINITY;
      to = fmaxf(to, m[j]);
    }
    const float mm = to == -INFINITY ? 0.0f : to, f0 = __builtin_amdgcn_exp2f(top - mm);
    top = to;
    sum *= f0;
#pragma unroll
    for (int b = 0; b < PB; ++b) o[b] *= f0;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const float f = __builtin_amdgcn_exp2f(m[j] - mm);   // 0 past the last part
      if (k0 + j * step >= p.count) continue;
      sum = __builtin_fmaf(f, l[j], sum);
#pragma unroll
      for (int b = 0; b < PB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b][e] = __builtin_fmaf(f, x[j][b][e], o[b][e]);
    }
  }
}
template <int WAVES>
struct JoinLds {
  float ml[WAVES][2][WAVE];
  f32x4 os[WAVES][WAVE];
};
template <typename T, int R, int DP, int WAVES>
__device__ __forceinline__ void join(const AttnArgs &a, int b, JoinLds<WAVES> &lds) {
  constexpr int ROWS = R > 32 ? 32 : 16, PER = ROWS * DP / 256, PB = PER < 4 ? PER : 4;
  auto &ml = lds.ml;
  auto &os = lds.os;
  const AttnPart p = a.rec[b];
  if (p.count == 0) return;
  const int share = b - p.w, shares = p.count - 1, wave = wave_id_u(), lane = lane_id();
  const int pieces = (p.n + ROWS - 1) / ROWS * PER;
  // (a row of the part past the unit's holds something, which is not stored)
  auto row = [&](int q) { return q / PER * ROWS + lane % ROWS; };
  if (R > 32 && p.count <= 4) {   // a wavefront several pieces
    for (int q0 = (share * WAVES + wave) * PB; q0 < pieces; q0 += shares * WAVES * PB) {
      float top, sum;
      f32x4 o[PB];
      join_sum<R, DP, PB, 2>(a, p, row(q0), q0, 0, 1, top, sum, o);
#pragma unroll
      for (int b = 0; b < PB; ++b) join_store<T, ROWS, DP>(a, p, row(q0), q0 + b, top, sum, o[b]);
    }
    return;
  }
  // `per` wavefronts a piece, with every so-manieth part
  int per = 1;
  while (per < WAVES && per * 8 < p.count) per *= 2;
  const int sub = wave & (per - 1), groups = WAVES / per, group = wave / per;
  for (int p0 = share * groups; p0 < pieces; p0 += shares * groups) {
    const int q = min(p0 + group, pieces - 1), r = row(q);
    float top, sum;
    f32x4 o[1];
    join_sum<R, DP, 1, 8>(a, p, r, q, sub, per, top, sum, o);
    if (per == 1) {
      if (p0 + group < pieces) join_store<T, ROWS, DP>(a, p, r, q, top, sum, o[0]);
      continue;
    }
    ml[wave][0][lane] = top;
    ml[wave][1][lane] = sum;
    os[wave][lane] = o[0];
    __syncthreads();
    if (sub == 0 && p0 + group < pieces) {
      float to = -INFINITY, t = 0.0f;
      for (int v = 0; v < per; ++v) to = fmaxf(to, ml[wave + v][0][lane]);
      const float mm = to == -INFINITY ? 0.0f : to;
      f32x4 x = {0, 0, 0, 0};
      for (int v = 0; v < per; ++v) {
        const float f = __builtin_amdgcn_exp2f(ml[wave + v][0][lane] - mm);
        t = __builtin_fmaf(f, ml[wave + v][1][lane], t);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(f, os[wave + v][lane][e], x[e]);
      }
      join_store<T, ROWS, DP>(a, p, r, q, to, t, x);
    }
    __syncthreads();
  }
}
template <typename T, int R, int DP>
__global__ __launch_bounds__(R > 32 ? 1024 : 512)
void k_attn_join(AttnArgs a) {
  __shared__ JoinLds<(R > 32 ? 16 : 8)> lds;
  join<T, R, DP>(a, blockIdx.x, lds);
}
// both kernels' in one launch
template <int RF, int RM, int DP>
__global__ __launch_bounds__(1024)
void k_attn_join_both(AttnArgs few, AttnArgs many) {
  __shared__ JoinLds<16> lds;
  if ((int)blockIdx.x < many.W) join<uint16_t, RM, DP>(many, blockIdx.x, lds);
  else join<uint16_t, RF, DP>(few, blockIdx.x - many.W, lds);
}

// The launches of a call.  Sequences of at most FEW_ROWS packed rows are k_attn_few's,
// longer ones (16-bit) k_attn_many's; where there may be both, both run, on parts of the
// workspace of their own, and one launch joins the units of both.  Calls whose products
// come to at most FEW_FLOPS are k_attn_few's alone, however long their sequences are: a
// unit of k_attn_many takes 9 us before its first block (its rows go through eight
// wavefronts' ring), and each launch about 4.  Measured, k_attn_few alone against
// k_attn_many or both, by what the products can come to: one sequence 1.6 GFLOP 23.4 against
// 25.8 us, 2.2 28.8 against 23.8; several 0.2 GFLOP 16.3 against 32.3, 1.4 23.7 against 34.6,
// 3.1 26.9 against 27.9, 10 67 against 45.6; at D 256, where its tiles are of 16 rows, one of
// 1.0 21.5 against 25.3, of 2.1 34.5 against 28.3.
constexpr int FEW_ROWS = 32;
constexpr double FEW_FLOPS = 3e9, FEW_FLOPS_ONE = 2e9, FEW_FLOPS_256 = 1e9;
// Units go to one workgroup each, with no parts and no join, where splitting them over the
// workgroups that there are would save few blocks of keys a workgroup: at tiles of 16 rows
// 6, 4 and 2.5 of heads of 64, 128 and 256 elements (a block takes 0.9, 1.4 and 1.9 us, a
// join 4 and the parts some), half as many at 32.  Of D 128, in parts and whole: 256 units of
// four blocks 18.6 and 13.9 us, of eight 22.9 and 19.3; 2048 of two 36.8 and 34.2; 32 of four
// 11.5 and 12.2, of eight (in parts by this rule) 12.4 and 17.7.  More units than workgroups
// only up to two blocks: 2048 of up to six (ragged) 38.8 and 53.
constexpr long long WHOLE_BLOCKS = 8;
// What a unit costs besides its blocks (queries, the ring's filling, the state's way out), in
// blocks, so that a workgroup with ends of three units has fewer blocks.  Without, and with
// these: 64 sequences of up to 8192 keys 63.1 and 56.8 us, 128 of up to 600 36.9 and 28.1,
// 200 of up to 1000 with heads of 256 153 and 97; chunks of 2048 tokens (32 heads on 8)
// 101 and 63.5, of 1000 54.2 and 39.5, of 2048 over 8191 keys 240 and 238.  Half and twice
// as much are within 5% of it, mostly slower.
constexpr int FEW_PAD = 2, MANY_PAD = 4;
struct Launch {
  int R, BK, W, coarse, pad;   // W 0: none
  uint32_t limit;           // of the line's length
  bool whole;
  size_t part, rec;         // in the workspace, bytes
};
struct Plan {
  int dp;
  Launch few, many;
  size_t bytes;
};
Plan plan(bool bf16, int D, int Hq, const KvCache &c, const KvBatch &b, long long rows, int window, int n_cu) {
  Plan p{};
  p.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const long long G = Hq / c.Hk, most = b.max_q * G;
  auto shape = [&](Launch &l, int R, int BK, int occ, int pad, double whole) {
    l.R = R;
    l.BK = BK;
    const long long blocks = (((long long)b.max_pages << c.shift) + BK - 1) / BK;
    // (what the rows come to; starts on the device that say more are not followed, see AttnWork)
    const double bound = (double)b.n_seq * c.Hk * ((most + R - 1) / R);
    double units = ((double)b.n_seq + (double)rows * G / R) * c.Hk;
    if (bound < units) units = bound;
    const double slots = (double)occ * n_cu;
    l.whole = units <= slots ? blocks <= WHOLE_BLOCKS && blocks * (1 - units / slots) <= whole * 16 / R
                             : whole > 0 && blocks <= 2;
    const auto length = [&] { return units * (double)((blocks >> l.coarse) + 1 + (pad >> l.coarse)); };
    while (length() > 1e9) ++l.coarse;
    l.pad = l.whole ? 0 : pad >> l.coarse;
    l.limit = (uint32_t)(l.whole ? units : length()) + 1;
    const double want = l.whole ? units : units * (blocks + pad);
    l.W = (int)(want < slots ? want : slots);
    l.part = p.bytes;
    if (!l.whole) p.bytes += 2 * (size_t)l.W * R * (p.dp + 2) * 4;
    l.rec = p.bytes = (p.bytes + 255) & ~(size_t)255;
    if (!l.whole) p.bytes += ((size_t)l.W * sizeof(AttnPart) + 255) & ~(size_t)255;
  };
  // (the lengths are on the device: this is the most that the products can come to)
  const double keys = (double)((long long)b.max_pages << c.shift), span = window > 0 ? (double)window + b.max_q : keys;
  const double flops = 4.0 * p.dp * Hq * rows * (span < keys ? span : keys);
  const bool small = !bf16 || most <= FEW_ROWS || flops <= (p.dp == 256 ? FEW_FLOPS_256 : b.n_seq == 1 ? FEW_FLOPS_ONE : FEW_FLOPS);
  // (tiles of 16 rows hold a token's heads: beside k_attn_many few sequences have more than
  // one; 17 sequences, one of them of 509 tokens: 56.4 us against 58.9 with tiles of 32)
  if (small || b.n_seq > 1) {
    const int R = p.dp == 256 || most <= 16 || (!small && bf16 && G <= 16) ? 16 : 32;
    shape(p.few, R, 64, few_occ(bf16, p.dp, R / 16), FEW_PAD, p.dp == 64 ? 6.0 : p.dp == 128 ? 4.0 : 2.5);
  }
  if (!small) shape(p.many, p.dp == 256 ? 128 : 256, p.dp == 256 ? 32 : 64, 1, MANY_PAD, -1.0);
  if (p.bytes == 0) p.bytes = 256;
  return p;
}

}  // namespace

size_t attn_ws_bytes(bool bf16, int D, int Hq, const KvCache &c, const KvBatch &b, long long rows,
                     int n_cu) {
  // (of any window: none, and the least)
  const size_t all = plan(bf16, D, Hq, c, b, rows, 0, n_cu).bytes, one = plan(bf16, D, Hq, c, b, rows, 1, n_cu).bytes;
  return all > one ? all : one;
}

hipError_t launch_attn(const AttnCall &call, const KvCache &c, const KvBatch &b, void *ws, int n_cu,
                       hipStream_t st) {
  const Plan p = plan(call.bf16, call.D, call.Hq, c, b, call.rows, call.window, n_cu);
  AttnArgs a{};
  a.q = call.q;
  a.o = call.o;
  a.lse = call.lse;
  a.c = c;
  a.b = b;
  a.rows = (int)call.rows;
  a.Hq = call.Hq;
  a.G = call.Hq / c.Hk;
  a.D = call.D;
  a.window = call.window;
  a.scale = call.scale * LOG2E;
  a.by_G = divisor(a.G);
  AttnArgs af = a, am = a;
  auto use = [&](AttnArgs &to, const Launch &l, int above, int upto) {
    to.above = above;
    to.upto = upto;
    to.W = l.W;
    to.whole = l.whole;
    to.coarse = l.coarse;
    to.limit = l.limit;
    to.pad = l.pad;
    to.by_W = divisor(l.W);
    to.part = reinterpret_cast<float *>(static_cast<char *>(ws) + l.part);
    to.rec = reinterpret_cast<AttnPart *>(static_cast<char *>(ws) + l.rec);
  };
  if (p.many.W) use(am, p.many, p.few.W ? FEW_ROWS : 0, 0x7FFFFFFF);
  if (p.few.W) use(af, p.few, 0, p.many.W ? FEW_ROWS : 0x7FFFFFFF);
#define BASE_MANY(DP)                                                                             \
  do {                                                                                            \
    launch_k(k_attn_many<DP>, dim3(p.many.W), dim3(ManyShape<DP>::THREADS), 0, st, am);           \
    if (!p.few.W || p.few.whole)                                                                  \
      launch_k(k_attn_join<uint16_t, ManyShape<DP>::R, DP>, dim3(p.many.W), dim3(1024), 0, st, am); \
  } while (0)
#define BASE_FEW(T, DP, NR)                                                                       \
  do {                                                                                            \
    launch_k(k_attn_few<T, DP, NR>, dim3(p.few.W), dim3(FewShape<T, DP, NR>::THREADS), 0, st, af); \
    if (p.few.whole) break;                                                                       \
    if (p.many.W)                                                                                 \
      launch_k(k_attn_join_both<16 * NR, ManyShape<DP>::R, DP>, dim3(p.few.W + p.many.W), dim3(1024), 0, st, af, am); \
    else                                                                                          \
      launch_k(k_attn_join<T, 16 * NR, DP>, dim3(p.few.W), dim3(512), 0, st, af);                 \
  } while (0)
#define BASE_FEW_R(T, DP)                                                                         \
  do { if (p.few.R == 16) BASE_FEW(T, DP, 1); else BASE_FEW(T, DP, 2); } while (0)
#define BASE_FEW_D(T)                                                                             \
  do {                                                                                            \
    if (p.dp == 64) BASE_FEW_R(T, 64);                                                            \
    else if (p.dp == 128) BASE_FEW_R(T, 128);                                                     \
    else BASE_FEW(T, 256, 1);                                                                     \
  } while (0)
  if (p.many.W) {
    if (p.dp == 64) BASE_MANY(64);
    else if (p.dp == 128) BASE_MANY(128);
    else BASE_MANY(256);
  }
  if (p.few.W) {
    if (call.bf16) BASE_FEW_D(uint16_t);
    else BASE_FEW_D(float);
  }
#undef BASE_FEW_D
#undef BASE_FEW_R
#undef BASE_FEW
#undef BASE_MANY
  return hipGetLastError();
}

}  // namespace basek
