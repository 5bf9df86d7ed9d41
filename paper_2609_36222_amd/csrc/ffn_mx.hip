// Grouped SwiGLU expert FFN on 4-bit weights (BASE_W_MXFP4): the same products as
// ffn.hip's, H[p] = bf16(silu(x . W_g) * (x . W_u)), pairbuf[p] = gate_p *
// (H[p] . W_d), with the weights' values e2m1 * 2^(s - 127) -- exact in bf16 --
// on MFMA 16x16x32 bf16, fp32 sums in ascending k.
//
// The activation's rounding.  Up to MX_TWO_B tokens h goes to the second product as a
// bf16 and an E5M2 part, h = hi + 2^-9 lo with lo = 2^9 (h - hi) rounded, so that its
// error is an eighth of a bf16 rounding's (as much as that where lo leaves E5M2's
// range, |h| < 2^-14 or > 57344): the launch is a weight stream, the scaled 16x16x128
// product takes the weights' codes and scales as they lie in memory, and the layer
// takes 2 to 4% longer.  Beyond, the matrix pipe is busy and the second part costs 7 to
// 20% of the layer (B = 256 57 -> 64 us, B = 1024 154 -> 181), so h is rounded to bf16, as in
// the 16-bit layers.  The output's error is then 1.4 times its own rounding's on average
// and, where few activations make it, up to 1.6; with both parts 1.0.
//
// The launch works on records {expert, first pair, pairs}: a slot (B <= 64) or
// a part of at most MX_NT 16-pair tiles of one, with their token lists, one copy
// per die.  A workgroup takes (record, row group): RW wavefronts side by side on
// T 16-row tiles each, and KW such rows of wavefronts on consecutive shares
// of the contraction, joined through LDS in ascending order -- a sum has
// one writer and one order.  Weights come to registers (16 bytes a lane: four
// operands and one scale, see mx.hpp) DT + 1 steps of 128 ahead, the token rows
// of up to NT tiles to an LDS ring of DT + 1 steps that the RW wavefronts share.
//
// What bounds it.  Few tokens: latency.  B = 1, 8 Qwen3-shaped slots, 13 MB of gate and
// up weights in 7.0 us, six steps of loads behind the launch, the records and the
// token list.  Beyond 32 tokens: the matrix pipe, the conversions in front of it and the
// token rows' way through LDS, in turn rather than at once.  B = 256, 32 slots:
// gate/up 24.4 us (530 TFLOP/s, 2.2 TB/s of weights), without its products 13.9,
// without either kind of loads 21; down 17.7, 4.5 of it the fp32 pair rows'
// stores.  Mixtral-shaped, B = 128, 4 slots: gate/up 83 to 91 (660 to 720 TFLOP/s),
// without products 21.6, without loads 64; down 52.
#include "common.hpp"
#include "ffn.hpp"
#include "internal.hpp"
#include "mx.hpp"

namespace basek {

// LO: the token rows have a second, 8-bit part (down)
template <int NT_, int T_, int RW_, int KW_, int DT_, bool LO_ = false>
struct MxShape {
  static constexpr int NT = NT_, T = T_, RW = RW_, KW = KW_, DT = DT_;
  static constexpr bool LO = LO_;
  static constexpr int WAVES = RW * KW, THREADS = WAVES * WAVE, RING = DT + 1;
  static constexpr int HL = (NT * 4 + RW - 1) / RW;    // loads per wavefront and step: bf16 rows
  static constexpr int LL = LO ? (NT * 2 + RW - 1) / RW : 0;   // ... the 8-bit parts
  static constexpr int TL = HL + LL;
  static constexpr int SLOT = NT * 4096 + LL * RW * 1024;      // a step's token rows
  static constexpr int SL = KW == 1 ? T : 2 * T;       // scale loads per four steps
  static constexpr int LDS = KW * RING * SLOT;
  static constexpr int GROUP = RW * T;                 // tiles per workgroup
  static constexpr int WPE = NT * T >= 16 ? 2 : DT == 1 ? 4 : 3;   // wavefronts per SIMD
  static_assert(DT + 1 < MX_CHUNK, "weights, one step further ahead, have a stage to spare");
  static_assert(LDS >= (KW > 1 ? WAVES * T * NT * 1024 : 0), "partial sums in the ring");
};

// The record and row group of this workgroup.  Workgroup b runs
// on die b % N_XCD; the row groups of slot `ord` are numbered on from the previous
// slot's and number v lies on die v % N_XCD, so that all parts of a slot read a
// row group's weights through one L2 and every die has its share of every slot.
// `shares` workgroups share a record's contraction.
struct MxPlan {
  int budget, ns, nrec, parts, shares;
  const SpRec *rec;
};
struct MxWork {
  int u, p0, n, rg, share;
};
template <bool SPLIT = false>
__device__ __forceinline__ MxWork mx_work(const MxPlan &pl, int RG) {
  const int die = blockIdx.x % N_XCD, q = blockIdx.x / N_XCD;
  const int shares = SPLIT ? pl.shares : 1, per = ((RG + N_XCD - 1) / N_XCD) * shares;
  const int y = q / per, zs = q - y * per, k = zs / shares;
  // slots: the shared experts first, they run for every token
  const int i = pl.parts ? y : (y < pl.ns ? pl.budget + y : y - pl.ns);
  const SpRec r = pl.rec[die * pl.nrec + i];
  const int ord = pl.parts ? __builtin_amdgcn_readfirstlane(r.pad) : y;
  const int rg = ((die - ord * RG) & (N_XCD - 1)) + N_XCD * k;
  return {__builtin_amdgcn_readfirstlane(r.u), __builtin_amdgcn_readfirstlane(r.p0),
          rg < RG ? __builtin_amdgcn_readfirstlane(r.n) : 0, rg, zs - k * shares};
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
// acc + the rows' codes and scale byte times 2^-9 times 128 E5M2 elements: lane (n, g)
// has the elements 16 g .. +15 and 64 + 16 g .. +15 of column n
__device__ __forceinline__ f32x4 mfma_lo(u32x4 codes, uint32_t byte, u32x4 lo0, u32x4 lo1, f32x4 acc) {
  const i32x8 a = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
  const i32x8 b = {(int)lo0[0], (int)lo0[1], (int)lo0[2], (int)lo0[3],
                   (int)lo1[0], (int)lo1[1], (int)lo1[2], (int)lo1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 1, 0, (int)byte, 0, 127 - 9);
}
// the E5M2 part of h beside its bf16 rounding, as fp32 for the conversion: within its
// range, 0 for NaN and infinities
__device__ __forceinline__ float mx_lo(float h, uint16_t hi) {
  const float v = 512.0f * (h - bf16_to_f32(hi));
  return v == v ? fminf(fmaxf(v, -57344.0f), 57344.0f) : 0.0f;
}

__device__ __forceinline__ int mx_block_pos(int g) { return (0x9C >> (2 * g)) & 3; }   // 0, 3, 1, 2
__device__ __forceinline__ int mx_block_at(int pos) { return (0x78 >> (2 * pos)) & 3; }  // its inverse

// The wait of a wavefront's step 4 i + p: until its tokens and, older, its weights
// are there.  Behind the tokens of step s are the tokens of s + 1 .. s + DT - 1
// (TL loads each) and the weights of s + 1 .. s + DT (T each, and SL scale loads
// with every fourth); at first, with the prologue's weights in front of all
// tokens, only the weights requested since.
template <typename M>
__device__ __forceinline__ void mx_wait(bool first, int p) {
#define BASE_MXW(P)                                                                             \
  case P:                                                                                       \
    if (P < M::DT && first)                                                                     \
      wait_vm<(M::DT - 1) * M::TL + P * M::T + (M::DT + P) / MX_CHUNK * M::SL>();               \
    else                                                                                        \
      wait_vm<(M::DT - 1) * M::TL + M::DT * M::T + (M::DT + P) / MX_CHUNK * M::SL>();           \
    break;
  switch (p) { BASE_MXW(0) BASE_MXW(1) BASE_MXW(2) BASE_MXW(3) }
#undef BASE_MXW
}

// This wavefront's tiles of a matrix of `tiles` tiles of K elements: [t0, t0 + T), all
// of them there or none (`tiles` is a multiple of T).
template <int T>
struct MxTiles {
  int t0;
  bool active;
  rsrc_t rw[T];
};
template <typename M>
__device__ __forceinline__ MxTiles<M::T> mx_tiles(const uint8_t *w, int rg, int tiles, int K) {
  MxTiles<M::T> m;
  m.t0 = (rg * M::RW + wave_id_u() % M::RW) * M::T;
  m.active = m.t0 < tiles;
  const size_t tb = mx_tile_bytes(K);
#pragma unroll
  for (int t = 0; t < M::T; ++t)
    m.rw[t] = make_rsrc(w + (size_t)(m.active ? m.t0 + t : 0) * tb, m.active ? (uint32_t)tb : 0u);
  return m;
}
// row groups of such a matrix
__host__ __device__ inline int mx_groups(int tiles, int group) { return (tiles + group - 1) / group; }

// acc[t][j] = sum over this wavefront's share of the K elements of tile t of the
// weights times token tile j (N of them).  Token rows: resource rx; rows(i) says at
// which byte row i starts (FFN_TOK_PAD: a row of zeros).
//  * LDS: row n of a tile at 256 n, operand f of its block g in the 16 bytes at
//    (4 mx_block_pos(g) + f) ^ n.  A 16-byte read takes 16 lanes at a time, the rows
//    0..3 and 12..15 of an even block with the rows 4..11 of the odd one after it
//    (or the other way round), so the two blocks' places have to differ by 12: with
//    4 g + f half of the cycles were conflicts (Qwen3-shaped gate/up, B = 1024, 128
//    experts 106 -> 95 us).  Behind them, row n of an 8-bit part at 128 n, its 16-byte
//    piece p at p ^ (n / 2).
//  * Order of the loads: in step s the tokens of step s + DT and the weights of step
//    s + DT + 1, so that the wait for a step's tokens covers its weights and leaves
//    those of the DT steps after it in flight.
template <typename M, int N, bool SPLIT = false, typename Rows>
__device__ __forceinline__ void mx_stream(uint8_t *lds, const MxTiles<M::T> &m, int K, rsrc_t rx,
                                          rsrc_t rlo, Rows rows, f32x4 (&acc)[M::T][N],
                                          int share = 0, int shares = 1) {
  constexpr int T = M::T, DT = M::DT, L = (4 * N + M::RW - 1) / M::RW;   // loads of four rows
  static_assert(L * M::RW <= 4 * M::NT, "token loads stay in their slot");
  const int w = wave_id_u(), lane = lane_id(), kq = w / M::RW, rw = w % M::RW;
  uint8_t *ring = lds + kq * (M::RING * M::SLOT);
  // this wavefront's steps [s0, s1) and those of the longest share: the KW rows', or
  // (SPLIT) the workgroup's among `shares` of them, in whole chunks
  static_assert(!SPLIT || M::KW == 1, "one way to share a contraction");
  const int S = mx_steps(K), C = mx_chunks(K);
  const int s0 = SPLIT ? share * C / shares * MX_CHUNK : kq * S / M::KW;
  const int s1 = SPLIT ? min((share + 1) * C / shares * MX_CHUNK, S) : (kq + 1) * S / M::KW;
  const int most = SPLIT ? s1 - s0 : (S + M::KW - 1) / M::KW;
  const uint32_t Kb = (uint32_t)K * 2u;
  // the rows this lane stages: of the step's 4 N quarter tiles (four rows each) the
  // RW wavefronts take one after another in turn; lane l row l / 16 of the quarter,
  // the 16 bytes in place l % 16 of the row
  uint32_t tv[L], pc[L];
  constexpr int LL = M::LO ? (2 * N + M::RW - 1) / M::RW : 0;   // half tiles (eight rows) of the 8-bit part
  static_assert(LL <= M::LL, "... in the slot");
  uint32_t lv[LL + 1], lc[LL + 1];
  // the ring's slots in turn, as running offsets: step i's to read and step i + DT's
  // to fill (a remainder in the addresses costs an add per LDS read)
  int fill = 0, read = 0;
  auto next = [](int &slot) { slot = slot == (M::RING - 1) * M::SLOT ? 0 : slot + M::SLOT; };
  auto tokens = [&](int i) {
    uint8_t *slot = ring + fill + rw * 1024;
    next(fill);
    const uint32_t al = (uint32_t)(s0 + i) * 128u;
    const uint32_t at = (uint32_t)(s0 + i) * 256u;
#pragma unroll
    for (int q = 0; q < L; ++q)
      load_lds(rx, slot + q * (M::RW * 1024),
               s0 + i < s1 && at + pc[q] < Kb ? tv[q] + at + pc[q] : FFN_TOK_PAD, 0);
#pragma unroll
    for (int q = 0; q < LL; ++q)
      load_lds(rlo, slot + M::NT * 4096 + q * (M::RW * 1024),
               s0 + i < s1 && al + lc[q] < (uint32_t)K ? lv[q] + al + lc[q] : FFN_TOK_PAD, 0);
  };
  u32x4 wt[MX_CHUNK][T];
  uint32_t sc[T], sn[T], sh[T];
  auto weights = [&](int p, int i) {
    const int s = s0 + i;
    // past the share: beyond the tile's resource, zero
    const uint32_t c0 = s < s1 ? (uint32_t)(s / MX_CHUNK) * MX_CHUNK_BYTES : FFN_TOK_PAD;
    const uint32_t at = c0 + 256u + (uint32_t)(s % MX_CHUNK) * 1024u;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (p == 0) {
        sn[t] = __builtin_amdgcn_raw_buffer_load_b32(m.rw[t], (int)(c0 + lane * 4), 0, 0);
        if (M::KW > 1)   // a share may begin inside a chunk
          sh[t] = __builtin_amdgcn_raw_buffer_load_b32(m.rw[t], (int)(c0 + MX_CHUNK_BYTES + lane * 4), 0, 0);
      }
      wt[p][t] = __builtin_bit_cast(u32x4, bload(m.rw[t], at + lane * 16, 0));
    }
  };
#pragma unroll
  for (int t = 0; t < T; ++t) {
    sc[t] = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[t][j] = f32x4{0, 0, 0, 0};
  }
  // the weights first: the token list is still on its way
#pragma unroll
  for (int p = 0; p <= DT; ++p) weights(p, p);
#pragma unroll
  for (int q = 0; q < L; ++q) {
    const int k = rw + M::RW * q, r = 4 * (k & 3) + (lane >> 4), at16 = (lane & 15) ^ r;
    pc[q] = 64u * (uint32_t)mx_block_at(at16 >> 2) + 16u * (uint32_t)(at16 & 3);
    tv[q] = rows(16 * (k >> 2) + r);
  }
#pragma unroll
  for (int q = 0; q < LL; ++q) {
    const int k = rw + M::RW * q, r = 8 * (k & 1) + (lane >> 3);
    lc[q] = 16u * (uint32_t)((lane & 7) ^ (r >> 1));
    const uint32_t v = rows(16 * (k >> 1) + r);
    lv[q] = v == FFN_TOK_PAD ? v : v / 2;   // half the bytes of the bf16 row
  }
#pragma unroll
  for (int p = 0; p < DT; ++p) tokens(p);
  const uint8_t *op[4];   // operand f of this lane's token and block, in slot 0
#pragma unroll
  for (int f = 0; f < 4; ++f)
    op[f] = ring + (lane & 15) * 256 + 16 * ((4 * mx_block_pos(lane >> 4) + f) ^ (lane & 15));
  const uint8_t *ol[2];   // the 8-bit part's halves
#pragma unroll
  for (int f = 0; f < 2; ++f)
    ol[f] = ring + M::NT * 4096 + (lane & 15) * 128 + 16 * ((4 * f + (lane >> 4)) ^ ((lane & 15) >> 1));
  for (int i0 = 0; i0 < most; i0 += MX_CHUNK) {
#pragma unroll
    for (int p = 0; p < MX_CHUNK; ++p) {
      const int i = i0 + p;
      mx_wait<MxShape<N, T, M::RW, M::KW, DT, M::LO>>(i0 == 0, p);
      if (M::RW > 1) wg_barrier();   // the others' rows are there, the next slot is read
      __builtin_amdgcn_sched_barrier(0);
      tokens(i + DT);
      weights((p + DT + 1) % MX_CHUNK, i + DT + 1);
      __builtin_amdgcn_sched_barrier(0);
      if (p == 0) {
#pragma unroll
        for (int t = 0; t < T; ++t)
          sc[t] = M::KW > 1 ? __builtin_amdgcn_alignbyte(sh[t], sn[t], (uint32_t)s0 & 3u) : sn[t];
      }
      if (m.active && s0 + i < s1) {
        float scale[T];
#pragma unroll
        for (int t = 0; t < T; ++t) scale[t] = mx_scale((sc[t] >> (8 * p)) & 0xFFu);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          bf16x8 x[N];
#pragma unroll
          for (int j = 0; j < N; ++j)
            x[j] = *reinterpret_cast<const bf16x8 *>(op[f] + read + j * 4096);
#pragma unroll
          for (int t = 0; t < T; ++t) {
            const bf16x8 a = mx_decode8(wt[p][t][f], scale[t]);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[t][j] = mfma16(a, x[j], acc[t][j]);
          }
        }
        if constexpr (M::LO) {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const u32x4 l0 = *reinterpret_cast<const u32x4 *>(ol[0] + read + j * 2048);
            const u32x4 l1 = *reinterpret_cast<const u32x4 *>(ol[1] + read + j * 2048);
#pragma unroll
            for (int t = 0; t < T; ++t)
              acc[t][j] = mfma_lo(wt[p][t], (sc[t] >> (8 * p)) & 0xFFu, l0, l1, acc[t][j]);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      next(read);
    }
  }
  wait_vm<0>();
  if constexpr (M::KW > 1) {   // the shares' sums into the ring
    wg_barrier();
    f32x4 *red = reinterpret_cast<f32x4 *>(lds) + w * (T * N * WAVE) + lane;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int j = 0; j < N; ++j) red[(t * N + j) * WAVE] = acc[t][j];
    __syncthreads();
  }
}

// out(t, j, sum) for the C tiles from t on at a time (gate/up: a gate tile and its up
// tile), each by one of the KW wavefronts that hold shares of them.
template <typename M, int N, int C, typename Out>
__device__ __forceinline__ void mx_emit(const uint8_t *lds, const f32x4 (&acc)[M::T][N], Out out) {
  if constexpr (M::KW == 1) {
#pragma unroll
    for (int t = 0; t < M::T; t += C)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        f32x4 v[C];
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = acc[t + c][j];
        out(t, j, v);
      }
  } else {
    const int w = wave_id_u(), kq = w / M::RW, rw = w % M::RW;
    const f32x4 *red = reinterpret_cast<const f32x4 *>(lds) + rw * (M::T * N * WAVE) + lane_id();
    for (int it = kq; it < M::T / C * N; it += M::KW) {
      const int t = it / N * C, j = it % N;
      f32x4 v[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        v[c] = red[((t + c) * N + j) * WAVE];
#pragma unroll
        for (int k = 1; k < M::KW; ++k) {
          const f32x4 o = red[(k * M::RW * M::T * N + (t + c) * N + j) * WAVE];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[c][q] = v[c][q] + o[q];
        }
      }
      out(t, j, v);
    }
  }
}

template <typename M>
__global__ __launch_bounds__(M::THREADS, M::WPE)
void k_mx_gateup(int d, int I, int E, MxPlan pl, int np, const uint8_t *__restrict__ w13r,
                 const uint8_t *__restrict__ w13s, const int32_t *__restrict__ sptok,
                 const uint16_t *__restrict__ x, int B, uint16_t *__restrict__ H,
                 uint8_t *__restrict__ Hlo) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[M::LDS];
  const MxWork k = mx_work(pl, mx_groups(I / 8, M::GROUP));
  const size_t eb = (size_t)(I / 8) * mx_tile_bytes(d);
  const uint8_t *w13 = k.u < E ? w13r + (size_t)k.u * eb : w13s + (size_t)(k.u - E) * eb;
  const rsrc_t rx = make_rsrc(x, (uint32_t)B * (uint32_t)d * 2u);
  const int lane = lane_id();
  // (more than once only for routes that name an expert twice: a shape's token tiles
  // hold a slot of its batches or a part)
  for (int c = 0; c < k.n; c += 16 * M::NT) {
    const int n = min(k.n - c, 16 * M::NT);
    const int32_t *tok = sptok + (size_t)(blockIdx.x % N_XCD) * np + k.p0 + c;
    uint16_t *h0 = H + (size_t)(k.p0 + c) * I;
    uint8_t *l0 = Hlo + (size_t)(k.p0 + c) * I;
    if (c > 0) wg_barrier();   // every wavefront is done with the ring
    sp_tiles<M::NT>((n + 15) / 16, [&](auto NC) {
      constexpr int N = decltype(NC)::value;
      const MxTiles<M::T> m = mx_tiles<M>(w13, k.rg, I / 8, d);
      f32x4 acc[M::T][N];
      mx_stream<M, N>(lds, m, d, rx, rx, [&](int i) {
        return i < n ? (uint32_t)tok[i] * (uint32_t)d * 2u : FFN_TOK_PAD;
      }, acc);
      if (!m.active) return;
      mx_emit<M, N, 2>(lds, acc, [&](int t, int j, const f32x4 (&v)[2]) {
        const int p = 16 * j + (lane & 15);
        if (p >= n) return;
        uint16_t h[4];
        float s[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          s[q] = silu_bf16(v[0][q]) * v[1][q];   // (silu within 2^-22)
          h[q] = f32_to_bf16(s[q]);
        }
        const u32x2 pk = {(uint32_t)h[0] | ((uint32_t)h[1] << 16),
                          (uint32_t)h[2] | ((uint32_t)h[3] << 16)};
        const size_t at = (size_t)p * I + 8 * (m.t0 + t) + 4 * (lane >> 4);
        *reinterpret_cast<u32x2 *>(h0 + at) = pk;
        if constexpr (M::NT < MX_NT) {   // up to MX_TWO_B tokens
          int lp = __builtin_amdgcn_cvt_pk_bf8_f32(mx_lo(s[0], h[0]), mx_lo(s[1], h[1]), 0, false);
          lp = __builtin_amdgcn_cvt_pk_bf8_f32(mx_lo(s[2], h[2]), mx_lo(s[3], h[3]), lp, true);
          *reinterpret_cast<int *>(l0 + at) = lp;
        }
      });
    });
  }
}

template <typename M, bool SPLIT>
__global__ __launch_bounds__(M::THREADS, M::WPE)
void k_mx_down(int d, int I, int E, MxPlan pl, const uint8_t *__restrict__ w2r,
               const uint8_t *__restrict__ w2s, const float *__restrict__ pair_gate,
               const uint16_t *__restrict__ H, const uint8_t *__restrict__ Hlo,
               float *__restrict__ pairbuf, size_t stride) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[M::LDS];
  const MxWork k = mx_work<SPLIT>(pl, mx_groups(d / 16, M::GROUP));
  const size_t eb = (size_t)(d / 16) * mx_tile_bytes(I);
  const uint8_t *w2 = k.u < E ? w2r + (size_t)k.u * eb : w2s + (size_t)(k.u - E) * eb;
  const int lane = lane_id();
  for (int c = 0; c < k.n; c += 16 * M::NT) {
    const int n = min(k.n - c, 16 * M::NT), p0 = k.p0 + c;
    const rsrc_t rx = make_rsrc(H + (size_t)p0 * I, (uint32_t)n * (uint32_t)I * 2u);
    const rsrc_t rlo = M::LO ? make_rsrc(Hlo + (size_t)p0 * I, (uint32_t)n * (uint32_t)I) : rx;
    float *out0 = pairbuf + (SPLIT ? k.share * stride : 0) + (size_t)p0 * d;
    if (c > 0) wg_barrier();
    sp_tiles<M::NT>((n + 15) / 16, [&](auto NC) {
      constexpr int N = decltype(NC)::value;
      const MxTiles<M::T> m = mx_tiles<M>(w2, k.rg, d / 16, I);
      float gt[N];
#pragma unroll
      for (int j = 0; j < N; ++j) gt[j] = pair_gate[p0 + min(16 * j + (lane & 15), n - 1)];
      f32x4 acc[M::T][N];
      mx_stream<M, N, SPLIT>(lds, m, I, rx, rlo, [&](int i) {
        return i < n ? (uint32_t)i * (uint32_t)I * 2u : FFN_TOK_PAD;
      }, acc, k.share, pl.shares);
      if (!m.active) return;
      mx_emit<M, N, 1>(lds, acc, [&](int t, int j, const f32x4 (&v)[1]) {
        const int p = 16 * j + (lane & 15);
        if (p >= n) return;
        float g = gt[0];
#pragma unroll
        for (int q = 1; q < N; ++q) g = j == q ? gt[q] : g;
        *reinterpret_cast<float4 *>(out0 + (size_t)p * d + 16 * (m.t0 + t) + 4 * (lane >> 4)) =
            float4{g * v[0][0], g * v[0][1], g * v[0][2], g * v[0][3]};
      });
    });
  }
}

// Down and the combine of few tokens (mx_few) in one launch: a workgroup
// owns 16 columns of y, goes over every slot and joins the pairs of each token in
// rank order, so that no pair rows go to memory and back.  A unit is (slot, share
// of the contraction), one wavefront's at a time; a wavefront goes over the chunks
// (four steps) of its units without a break, each step's registers and LDS rows
// refilled from the next chunk as soon as they have been read.  Token rows are
// staged four at a time, 256 contiguous bytes of each, and only as many as the
// batch has (RL loads of four rows): gathered in the operand's own order, 64
// scattered pieces a load, they took three times as long as the weights (24 slots,
// B = 5, 16.4 us).  The sums go to LDS by pair, and
// y_t = residual_t + sum_j gate_j o_j from there.  `shares` > 1 only where few
// slots would leave wavefronts without work.  The pairs' gates and places, which
// another die wrote, come straight into LDS behind the first chunk's loads.
constexpr int MXF_WAVES = 16;
constexpr int MXF_LDS = 148 << 10, MXF_SUMS = 24 << 10;   // dynamic LDS, the sums' part of it
constexpr int MXF_PAIRS = 512;   // pairs' places and gates in LDS, a multiple of 256
static_assert(MX_FEW_B * (MAX_K + MAX_SHARED) <= MXF_PAIRS, "the pairs of a batch");
static_assert(MX_FEW_B * (MAX_K + MAX_SHARED) * 16 * 4 <= MXF_SUMS, "one share's sums");
struct MxFewTail {
  int B, kc, shares;
  const int32_t *pair_of;
  const float *pair_gate;
  const void *residual;
  void *y;
};
struct MxItem {   // a chunk of a unit's pairs from c on, 4 RL at a time
  int k, u, p0, n, c, ch, ch1;
};
template <int RL>
__global__ __launch_bounds__(MXF_WAVES * WAVE)
void k_mx_down_combine(int d, int I, int E, int slots, MxPlan pl, MxFewTail tl,
                       const uint8_t *__restrict__ w2r, const uint8_t *__restrict__ w2s,
                       const uint16_t *__restrict__ H, const uint8_t *__restrict__ Hlo) {
  constexpr int LL = (RL + 1) / 2, STEP = (RL + LL) * 1024;   // loads of the 8-bit part; a step's rows
  // the sums [share][pair][16], then every wavefront's token rows of four steps
  extern __shared__ __attribute__((aligned(16))) float sums[];
  __shared__ __attribute__((aligned(16))) int pair_s[MXF_PAIRS];
  __shared__ __attribute__((aligned(16))) float gate_s[MXF_PAIRS];
  __shared__ __attribute__((aligned(16))) SpRec rec_s[MAX_SLOTS];
  const int w = wave_id_u(), lane = lane_id(), nw = (int)blockDim.x / WAVE;
  const int np = tl.B * tl.kc, tile = blockIdx.x, nu = (slots + pl.ns) * tl.shares;
  const SpRec *rec = pl.rec + (size_t)(blockIdx.x % N_XCD) * pl.nrec;
  for (int y = threadIdx.x; y < slots + pl.ns; y += blockDim.x)
    rec_s[y] = rec[y < pl.ns ? pl.budget + y : y - pl.ns];
  __syncthreads();
  const size_t tb = mx_tile_bytes(I), eb = (size_t)(d / 16) * tb;
  const int S = mx_steps(I), C = mx_chunks(I);
  const uint32_t Ib = (uint32_t)I * 2u;
  // the item after `it`: its next chunk, the unit's next pairs, the next unit
  // (k >= nu: none); shares in whole chunks, a chunk's scales with its steps
  auto unit = [&](MxItem &it) {
    for (; it.k < nu; it.k += nw) {
      const int y = it.k / tl.shares, q = it.k - y * tl.shares;
      const SpRec r = rec_s[y];
      it.n = __builtin_amdgcn_readfirstlane(r.n);
      it.ch = q * C / tl.shares;
      it.ch1 = (q + 1) * C / tl.shares;
      if (it.n <= 0) continue;
      it.u = __builtin_amdgcn_readfirstlane(r.u);
      it.p0 = __builtin_amdgcn_readfirstlane(r.p0);
      it.c = 0;
      return;
    }
  };
  auto next = [&](MxItem it) {
    if (++it.ch < it.ch1) return it;
    const int q = it.k % tl.shares;
    it.ch = q * C / tl.shares;
    if ((it.c += 4 * RL) < it.n) return it;
    it.k += nw;
    unit(it);
    return it;
  };
  uint8_t *ring = reinterpret_cast<uint8_t *>(sums + tl.shares * np * 16) + w * (MX_CHUNK * STEP);
  const int tok = lane & 15, g = lane >> 4;
  // (a row past the staged ones repeats one of them, in a column nobody reads)
  const uint8_t *op[4];
#pragma unroll
  for (int f = 0; f < 4; ++f)
    op[f] = ring + (tok % (4 * RL)) * 256 + 16 * ((4 * mx_block_pos(g) + f) ^ (tok % (4 * RL)));
  uint32_t pc[RL], rb[RL];   // this lane's piece and row of each load
#pragma unroll
  for (int q = 0; q < RL; ++q) {
    const int r = 4 * q + (lane >> 4), at16 = (lane & 15) ^ r;
    pc[q] = 64u * (uint32_t)mx_block_at(at16 >> 2) + 16u * (uint32_t)(at16 & 3);
    rb[q] = (uint32_t)r * Ib;   // rows past the slot's pairs are past rx: zeros
  }
  uint32_t lc[LL], lb[LL];
#pragma unroll
  for (int q = 0; q < LL; ++q) {
    const int r = 8 * q + (lane >> 3);
    lc[q] = 16u * (uint32_t)((lane & 7) ^ (r >> 1));
    lb[q] = (uint32_t)r * (uint32_t)I;
  }
  const uint8_t *ol[2];
#pragma unroll
  for (int f = 0; f < 2; ++f)
    ol[f] = ring + RL * 1024 + (tok % (8 * LL)) * 128 + 16 * ((4 * f + g) ^ ((tok % (8 * LL)) >> 1));
  u32x4 a[MX_CHUNK];
  uint32_t sn = 0;
  rsrc_t rw = make_rsrc(w2r, 0), rx = make_rsrc(H, 0), rlo = rx;
  auto request = [&](const MxItem &it, int p) {
    const bool have = it.k < nu;
    if (p == 0 && have) {
      const uint8_t *m = it.u < E ? w2r + (size_t)it.u * eb : w2s + (size_t)(it.u - E) * eb;
      rw = make_rsrc(m + tile * tb, (uint32_t)tb);
      const int n = min(it.n - it.c, 4 * RL);
      rx = make_rsrc(H + (size_t)(it.p0 + it.c) * I, (uint32_t)n * Ib);
      rlo = make_rsrc(Hlo + (size_t)(it.p0 + it.c) * I, (uint32_t)(n * I));
    }
    const int s = it.ch * MX_CHUNK + p;
    const uint32_t c0 = have && s < S ? (uint32_t)it.ch * MX_CHUNK_BYTES : FFN_TOK_PAD;
    if (p == 0) sn = __builtin_amdgcn_raw_buffer_load_b32(rw, (int)(c0 + lane * 4), 0, 0);
    a[p] = __builtin_bit_cast(u32x4, bload(rw, c0 + 256u + (uint32_t)p * 1024u + lane * 16, 0));
    const uint32_t at = (uint32_t)s * 256u;
#pragma unroll
    for (int q = 0; q < RL; ++q)
      load_lds(rx, ring + p * STEP + q * 1024, have && at + pc[q] < Ib ? rb[q] + at + pc[q] : FFN_TOK_PAD, 0);
    const uint32_t al = (uint32_t)s * 128u;
#pragma unroll
    for (int q = 0; q < LL; ++q)
      load_lds(rlo, ring + p * STEP + (RL + q) * 1024,
               have && al + lc[q] < (uint32_t)I ? lb[q] + al + lc[q] : FFN_TOK_PAD, 0);
  };
  MxItem it{w, 0, 0, 0, 0, 0, 0};
  unit(it);
#pragma unroll
  for (int p = 0; p < MX_CHUNK; ++p) request(it, p);
  if (w == 0) {
    const rsrc_t rp = make_rsrc(tl.pair_of, (uint32_t)np * 4u), rg = make_rsrc(tl.pair_gate, (uint32_t)np * 4u);
#pragma unroll
    for (int i = 0; i < MXF_PAIRS / 256; ++i) {
      load_lds(rp, pair_s + 256 * i, 1024u * i + lane * 16, 0);
      load_lds(rg, gate_s + 256 * i, 1024u * i + lane * 16, 0);
    }
  }
  f32x4 acc = {0, 0, 0, 0};
  while (it.k < nu) {
    const MxItem nx = next(it);
    const uint32_t sc = sn;
#pragma unroll
    for (int p = 0; p < MX_CHUNK; ++p) {
      // behind this step are three others, one of them with its chunk's scales
      // unless this step came with its own
      if (p == 0) wait_vm<3 * (1 + RL + LL)>();
      else wait_vm<3 * (1 + RL + LL) + 1>();
      __builtin_amdgcn_sched_barrier(0);
      const float scale = mx_scale((sc >> (8 * p)) & 0xFFu);
      bf16x8 x[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) x[f] = *reinterpret_cast<const bf16x8 *>(op[f] + p * STEP);
      const u32x4 l0 = *reinterpret_cast<const u32x4 *>(ol[0] + p * STEP);
      const u32x4 l1 = *reinterpret_cast<const u32x4 *>(ol[1] + p * STEP);
#pragma unroll
      for (int f = 0; f < 4; ++f) acc = mfma16(mx_decode8(a[p][f], scale), x[f], acc);
      acc = mfma_lo(a[p], (sc >> (8 * p)) & 0xFFu, l0, l1, acc);
      __builtin_amdgcn_sched_barrier(0);
      request(nx, p);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (it.ch + 1 == it.ch1) {
      if (tok < min(it.n - it.c, 4 * RL))
        *reinterpret_cast<f32x4 *>(sums + ((it.k % tl.shares) * np + it.p0 + it.c + tok) * 16 + 4 * g) = acc;
      acc = f32x4{0, 0, 0, 0};
    }
    it = nx;
  }
  wait_vm<0>();   // the pairs' places
  __syncthreads();
  for (int i = threadIdx.x; i < tl.B * 16; i += blockDim.x) {
    const int t = i >> 4, r = i & 15;
    const size_t o = (size_t)t * d + 16 * tile + r;
    float v = tl.residual ? bf16_to_f32(static_cast<const uint16_t *>(tl.residual)[o]) : 0.0f;
    for (int j = 0; j < tl.kc; ++j) {
      const int p = pair_s[t * tl.kc + j];
      if (p < 0) continue;   // a routed rank the token does not execute
      float e = sums[p * 16 + r];
      for (int q = 1; q < tl.shares; ++q) e = e + sums[(q * np + p) * 16 + r];
      v = v + gate_s[p] * e;
    }
    static_cast<uint16_t *>(tl.y)[o] = f32_to_bf16(v);
  }
}

// ----------------------------------------------------------------- launch --
namespace {
// The shapes by batch.  Up to 16 tokens a slot has one token tile and the launch is a
// weight stream whose latency counts: four wavefronts side by side, or, where
// that leaves gate/up with fewer workgroups than compute units, two and two on
// halves of the contraction (us, Qwen3-shaped gate/up, 8 slots at B = 1 and 10 at
// B = 16, 96 and 120 workgroups: 8.3 and 9.6 against 6.9 and 7.7; OLMoE-shaped,
// 24 slots at B = 5, 384 workgroups: 12.0 against 12.5; down, whose contraction is
// short: 5.2, 5.2 and 7.8 against 5.0, 6.0 and 8.4).  Past 32 tokens the matrix
// pipe is busy for most of the time, and more workgroups per CU pay more than
// deeper rings (DT = 1, 2, 3 at B = 256, 32 experts, gate/up 24.3, 24.9 and 30.1,
// down 17.6, 18.4 and 21.3).  With enough workgroups eight wavefronts share the
// token rows instead of four, which halves their traffic (gate/up, B = 1024, 128
// experts: 85 -> 77; 448 workgroups of Mixtral's shape 89 -> 81; but 192 at B = 256
// 24.7 -> 27.5, and 220 of Qwen1.5-MoE's shape at B = 61 17.8 -> 21.4; down, of short
// contractions, 52.8 and 52.9 at B = 1024, and 17.7 -> 19.2 at B = 256).  The line counts
// the workgroups of slots and full parts, which the host knows.
// (a shape's token tiles hold every slot of its batches: B <= 16, MX_TWO_B, FFN_SPLIT_B,
// or a part)
static_assert(MX_TWO_B == 32, "MxMid's token tiles");
using MxFew = MxShape<1, 2, 4, 1, 2>;
using MxFewSplit = MxShape<1, 2, 2, 2, 2>;
using MxMid = MxShape<2, 2, 4, 1, 2>;
using MxMany = MxShape<MX_NT, 2, 4, 1, 1>;
using MxManyWide = MxShape<MX_NT, 2, 8, 1, 1>;
using MxFewDown = MxShape<1, 2, 4, 1, 2, true>;
using MxMidDown = MxShape<2, 2, 4, 1, 2, true>;

// workgroups: records times row groups (the same number on every die) times the
// shares of a contraction
dim3 mx_grid(int recs, int RG, int shares) {
  return dim3((unsigned)(N_XCD * recs * ((RG + N_XCD - 1) / N_XCD) * shares));
}
}  // namespace

hipError_t launch_mx_gateup(const void *x, int B, int d, int I, int E, int K, int budget, int slots,
                            int ns, const void *w13, const void *w13s, const SpRec *rec,
                            const int32_t *sptok, void *H, void *Hlo, int n_cu, hipStream_t st) {
  const bool parts = mx_parts(B);
  const int nrec = mx_records(B, K, budget, ns);
  auto go = [&](auto shape) {
    using M = decltype(shape);
    launch_k(k_mx_gateup<M>, mx_grid(parts ? nrec : slots + ns, mx_groups(I / 8, M::GROUP), 1),
             dim3(M::THREADS), 0, st, d, I, E, MxPlan{budget, ns, nrec, (int)parts, 1, rec},
             B * (K + ns), (const uint8_t *)w13, (const uint8_t *)w13s, sptok, (const uint16_t *)x,
             B, (uint16_t *)H, (uint8_t *)Hlo);
  };
  static_assert(MxFew::GROUP == MX_GU_GROUP && MxFewSplit::GROUP <= MX_GU_GROUP &&
                    MxManyWide::GROUP == MX_GU_WIDE,
                "mx_gateup_shape's row groups");
  switch (mx_gateup_shape(B, I, K, budget, ns, n_cu)) {
    case MX_GU_FEW: go(MxFew{}); break;
    case MX_GU_FEW_SPLIT: go(MxFewSplit{}); break;
    case MX_GU_MID: go(MxMid{}); break;
    case MX_GU_MANY: go(MxMany{}); break;
    case MX_GU_MANY_WIDE: go(MxManyWide{}); break;
  }
  return hipGetLastError();
}

hipError_t launch_mx_down(int B, int d, int I, int E, int K, int budget, int slots, int ns,
                          const void *w2, const void *w2s, const SpRec *rec, const float *pair_gate,
                          const void *H, const void *Hlo, float *pairbuf, int shares,
                          hipStream_t st) {
  const bool parts = mx_parts(B);
  const int nrec = mx_records(B, K, budget, ns);
  auto go = [&](auto shape) {
    using M = decltype(shape);
    static_assert(M::GROUP == MX_DOWN_GROUP && M::KW == 1, "mx_down_shares");
    launch_k(shares > 1 ? k_mx_down<M, true> : k_mx_down<M, false>,
             mx_grid(parts ? nrec : slots + ns, mx_groups(d / 16, M::GROUP), shares),
             dim3(M::THREADS), 0, st, d, I, E,
             MxPlan{budget, ns, nrec, (int)parts, shares, rec}, (const uint8_t *)w2,
             (const uint8_t *)w2s, pair_gate, (const uint16_t *)H, (const uint8_t *)Hlo, pairbuf,
             (size_t)B * (K + ns) * d);
  };
  if (B <= 16) go(MxFewDown{});
  else if (B <= MX_TWO_B) go(MxMidDown{});
  else go(MxMany{});
  return hipGetLastError();
}

hipError_t launch_mx_down_combine(int B, int d, int I, int E, int K, int budget, int slots, int ns,
                                  const void *w2, const void *w2s, const SpRec *rec,
                                  const int32_t *pair_of, const float *pair_gate, const void *H,
                                  const void *Hlo, const void *residual, void *y, hipStream_t st) {
  const int units = mx_kept(B, K, budget) + ns, C = mx_chunks(I);
  const int bytes = B * (K + ns) * 16 * (int)sizeof(float);   // a share's sums
  const int rl = mx_row_loads(B);                             // loads of four rows a step
  const int ring = MX_CHUNK * (rl + (rl + 1) / 2) * 1024;     // a wavefront's token rows
  const int fit = (MXF_LDS - MXF_SUMS) / ring, waves = fit < MXF_WAVES ? fit : MXF_WAVES;
  int shares = waves / units;
  for (const int most : {C, MXF_SUMS / bytes})
    if (shares > most) shares = most;
  if (shares < 1) shares = 1;
  const int work = (slots + ns) * shares, nw = work < waves ? work : waves;
  const auto kern = rl == 1   ? k_mx_down_combine<1>
                    : rl == 2 ? k_mx_down_combine<2>
                              : k_mx_down_combine<4>;
  launch_k(kern, dim3(d / 16), dim3(WAVE * nw), (uint32_t)(shares * bytes + nw * ring), st, d, I, E,
           slots, MxPlan{budget, ns, budget + ns, 0, 1, rec},
           MxFewTail{B, K + ns, shares, pair_of, pair_gate, residual, y}, (const uint8_t *)w2,
           (const uint8_t *)w2s, (const uint16_t *)H, (const uint8_t *)Hlo);
  return hipGetLastError();
}

}  // namespace basek
