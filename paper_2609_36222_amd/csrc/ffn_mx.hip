// Grouped SwiGLU expert FFN on 4-bit weights (BASE_W_MXFP4): the same products as
// ffn.hip's, H[p] = bf16(silu(x . W_g) * (x . W_u)), pairbuf[p] = gate_p *
// (H[p] . W_d), with the weights' values e2m1 * 2^(s - 127) -- exact in bf16 --
// on MFMA 16x16x32 bf16, fp32 sums in ascending k.  The activation H is rounded to
// bf16 for the second product, as in the 16-bit layers.
//
// The launch works on records {expert, first pair, pairs}: a slot (B <= 64) or
// a part of at most MX_NT 16-pair tiles of one, with their token lists, one copy
// per die.  A workgroup takes (record, row group); its wavefronts own MX_T
// 16-row tiles each over the whole contraction, so a sum has one writer and one
// order.  Weights come to registers (16 bytes a lane: four operands and one
// scale, see mx.hpp), MX_DW steps of 128 ahead; the record's token rows are
// staged through an LDS ring that the wavefronts share.
#include "common.hpp"
#include "ffn.hpp"
#include "internal.hpp"
#include "mx.hpp"

namespace basek {

constexpr int MX_WAVES = 4;
constexpr int MX_THREADS = MX_WAVES * WAVE;
constexpr int MX_T = 2;    // tiles per wavefront (gate/up: a gate tile and its up tile)
constexpr int MX_DW = 4;   // steps of weights in flight (a chunk: the stage index is static)
constexpr int MX_DT = MX_DW - 1;   // steps of tokens in flight
constexpr int MX_RING = MX_DT + 1;
static_assert(MX_DW == MX_CHUNK, "one chunk of stages");

// The record and row group of this workgroup.  Workgroup b runs on die b %
// N_XCD; the row groups of slot `ord` are numbered on from the previous slot's
// and number v lies on die v % N_XCD, so that all parts of a slot read a row
// group's weights through one L2 and every die has its share of every slot.
struct MxWork {
  int u, p0, n, rg;
};
__device__ __forceinline__ MxWork mx_work(int budget, int ns, int nrec, bool parts, int RG,
                                          const SpRec *__restrict__ rec) {
  const int die = blockIdx.x % N_XCD, q = blockIdx.x / N_XCD;
  const int per = (RG + N_XCD - 1) / N_XCD;
  const int y = q / per, k = q - y * per;
  // slots: the shared experts first, they run for every token
  const int i = parts ? y : (y < ns ? budget + y : y - ns);
  const SpRec r = rec[die * nrec + i];
  const int ord = parts ? __builtin_amdgcn_readfirstlane(r.pad) : y;
  const int rg = ((die - ord * RG) & (N_XCD - 1)) + N_XCD * k;
  return {__builtin_amdgcn_readfirstlane(r.u), __builtin_amdgcn_readfirstlane(r.p0),
          rg < RG ? __builtin_amdgcn_readfirstlane(r.n) : 0, rg};
}

// acc[t][j] = sum over the K elements of tile t of the weights (resource rw[t])
// times token tile j.  Token rows:
// resource rx, this lane's row of tile j at byte tv[j] (FFN_TOK_PAD or more: a
// zero row); it stages one 16-byte piece of the 256 a step has of the row.
//  * LDS: row n of a tile at 256 n, its piece p at position p ^ n, so that
//    neither the 16 rows' reads of one piece nor a row's write meet a bank twice.
//  * Order of the loads: in iteration s the tokens of step s + MX_DT, then the
//    weights of step s + MX_DW (with a chunk's first step, that chunk's scales).
//    So when the tokens of step s have arrived, so have its weights, and the
//    weights of the three steps after it may still be in flight.
template <int NT>
__device__ __forceinline__ void mx_stream(uint8_t *ring, const rsrc_t (&rw)[MX_T], int K,
                                          rsrc_t rx, const uint32_t (&tv)[NT],
                                          f32x4 (&acc)[MX_T][NT]) {
  const int w = wave_id_u(), lane = lane_id();
  const int S = mx_steps(K);
  const int row = 4 * w + (lane >> 4);                       // of a tile, staged by this lane
  const uint32_t pc = 16u * (uint32_t)((lane & 15) ^ row);   // its piece, in bytes of the step
  const uint32_t Kb = (uint32_t)K * 2u;
  const int n = lane & 15, g = lane >> 4;
  auto tokens = [&](int s) {
    uint8_t *slot = ring + (s % MX_RING) * (NT * 4096) + w * 1024;
    const uint32_t at = (uint32_t)s * 256u + pc;
#pragma unroll
    for (int j = 0; j < NT; ++j) load_lds(rx, slot + j * 4096, at < Kb ? tv[j] + at : FFN_TOK_PAD, 0);
  };
  u32x4 wt[MX_DW][MX_T];
  uint32_t sc[MX_T], sn[MX_T];
  auto weights = [&](int p, int s) {
    // past the tile: beyond its resource, zero
    const uint32_t c0 = s < S ? (uint32_t)(s / MX_CHUNK) * MX_CHUNK_BYTES : FFN_TOK_PAD;
#pragma unroll
    for (int t = 0; t < MX_T; ++t) {
      if (p == 0) sn[t] = __builtin_amdgcn_raw_buffer_load_b32(rw[t], (int)(c0 + lane * 4), 0, 0);
      wt[p][t] = __builtin_bit_cast(u32x4, bload(rw[t], c0 + 256u + (uint32_t)p * 1024u + lane * 16, 0));
    }
  };
#pragma unroll
  for (int t = 0; t < MX_T; ++t)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[t][j] = f32x4{0, 0, 0, 0};
  // the groups of iterations -DW .. -1
  weights(0, 0);
#pragma unroll
  for (int p = 0; p < MX_DT; ++p) {
    tokens(p);
    weights(p + 1, p + 1);
  }
#pragma unroll
  for (int t = 0; t < MX_T; ++t) sc[t] = 0;
  for (int s0 = 0; s0 < S; s0 += MX_DW) {
#pragma unroll
    for (int p = 0; p < MX_DW; ++p) {
      const int s = s0 + p;
      // in flight: the tokens of s + 1, s + 2 and the weights of s + 1 .. s + 3, one
      // of which starts a chunk unless this step does
      if (p == 0) wait_vm<2 * NT + 3 * MX_T>();
      else wait_vm<2 * NT + 4 * MX_T>();
      wg_barrier();
      __builtin_amdgcn_sched_barrier(0);
      tokens(s + MX_DT);
      __builtin_amdgcn_sched_barrier(0);
      if (p == 0) {
#pragma unroll
        for (int t = 0; t < MX_T; ++t) sc[t] = sn[t];
      }
      if (s < S) {
        const uint8_t *sb = ring + (s % MX_RING) * (NT * 4096) + n * 256;
        float scale[MX_T];
#pragma unroll
        for (int t = 0; t < MX_T; ++t) scale[t] = mx_scale((sc[t] >> (8 * p)) & 0xFFu);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          bf16x8 x[NT];
#pragma unroll
          for (int j = 0; j < NT; ++j)
            x[j] = *reinterpret_cast<const bf16x8 *>(sb + j * 4096 + 16 * ((4 * g + f) ^ n));
#pragma unroll
          for (int t = 0; t < MX_T; ++t) {
            const bf16x8 a = mx_decode8(wt[p][t][f], scale[t]);
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[t][j] = mfma16(a, x[j], acc[t][j]);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      weights(p, s + MX_DW);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  wait_vm<0>();
}

// this lane's staged row of token tile j: pair 16 j + row
__device__ __forceinline__ int mx_stage_row(int j) { return 16 * j + 4 * wave_id() + (lane_id() >> 4); }

template <int NT>
__device__ __forceinline__ void mx_gateup_part(uint8_t *ring, const MxWork &k, int d, int I,
                                               const uint8_t *__restrict__ w13, const int32_t *tok,
                                               int n, rsrc_t rx, uint16_t *__restrict__ h0) {
  const int w = wave_id_u(), lane = lane_id();
  const int r = k.rg * MX_WAVES + w;   // row-pair tile: I / 16 is a multiple of MX_WAVES
  const size_t tb = mx_tile_bytes(d);
  rsrc_t rw[MX_T];
#pragma unroll
  for (int t = 0; t < MX_T; ++t) rw[t] = make_rsrc(w13 + (size_t)(2 * r + t) * tb, (uint32_t)tb);
  uint32_t tv[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int i = mx_stage_row(j);
    tv[j] = i < n ? (uint32_t)tok[i] * (uint32_t)d * 2u : FFN_TOK_PAD;
  }
  f32x4 acc[MX_T][NT];
  mx_stream<NT>(ring, rw, d, rx, tv, acc);
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int p = 16 * j + (lane & 15);
    if (p < n) {
      uint16_t h[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) h[q] = f32_to_bf16(silu_bf16(acc[0][j][q]) * acc[1][j][q]);
      const u32x2 pk = {(uint32_t)h[0] | ((uint32_t)h[1] << 16),
                        (uint32_t)h[2] | ((uint32_t)h[3] << 16)};
      *reinterpret_cast<u32x2 *>(h0 + (size_t)p * I + 16 * r + 4 * (lane >> 4)) = pk;
    }
  }
}

template <int NT>
__global__ __launch_bounds__(MX_THREADS)
void k_mx_gateup(int d, int I, int E, int budget, int ns, int nrec, int parts, int np,
                 const uint8_t *__restrict__ w13r, const uint8_t *__restrict__ w13s,
                 const SpRec *__restrict__ rec, const int32_t *__restrict__ sptok,
                 const uint16_t *__restrict__ x, int B, uint16_t *__restrict__ H) {
  __shared__ __attribute__((aligned(16))) uint8_t ring[MX_RING * NT * 4096];
  const MxWork k = mx_work(budget, ns, nrec, parts != 0, I / 16 / MX_WAVES, rec);
  if (k.n <= 0) return;
  const size_t eb = (size_t)(I / 8) * mx_tile_bytes(d);
  const uint8_t *w13 = k.u < E ? w13r + (size_t)k.u * eb : w13s + (size_t)(k.u - E) * eb;
  const int32_t *tok = sptok + (size_t)(blockIdx.x % N_XCD) * np + k.p0;
  const rsrc_t rx = make_rsrc(x, (uint32_t)B * (uint32_t)d * 2u);
  for (int c = 0; c < k.n; c += 16 * NT) {
    const int n = min(k.n - c, 16 * NT);
    if (c > 0) wg_barrier();   // every wavefront is done with the ring
    sp_tiles<NT>((n + 15) / 16, [&](auto N) {
      mx_gateup_part<decltype(N)::value>(ring, k, d, I, w13, tok + c, n, rx,
                                         H + (size_t)(k.p0 + c) * I);
    });
  }
}

template <int NT>
__device__ __forceinline__ void mx_down_part(uint8_t *ring, const MxWork &k, int d, int I,
                                             const uint8_t *__restrict__ w2,
                                             const uint16_t *__restrict__ h0, int n,
                                             const float *__restrict__ gate0,
                                             float *__restrict__ out0) {
  const int w = wave_id_u(), lane = lane_id();
  const int r = (k.rg * MX_WAVES + w) * MX_T;   // d / 16 is a multiple of MX_WAVES MX_T
  const size_t tb = mx_tile_bytes(I);
  rsrc_t rw[MX_T];
#pragma unroll
  for (int t = 0; t < MX_T; ++t) rw[t] = make_rsrc(w2 + (size_t)(r + t) * tb, (uint32_t)tb);
  const rsrc_t rx = make_rsrc(h0, (uint32_t)n * (uint32_t)I * 2u);
  float gt[NT];
  uint32_t tv[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int i = mx_stage_row(j);
    tv[j] = i < n ? (uint32_t)i * (uint32_t)I * 2u : FFN_TOK_PAD;
    gt[j] = gate0[min(16 * j + (lane & 15), n - 1)];
  }
  f32x4 acc[MX_T][NT];
  mx_stream<NT>(ring, rw, I, rx, tv, acc);
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int p = 16 * j + (lane & 15);
    if (p < n) {
#pragma unroll
      for (int t = 0; t < MX_T; ++t) {
        const f32x4 o = acc[t][j];
        *reinterpret_cast<float4 *>(out0 + (size_t)p * d + 16 * (r + t) + 4 * (lane >> 4)) =
            float4{gt[j] * o[0], gt[j] * o[1], gt[j] * o[2], gt[j] * o[3]};
      }
    }
  }
}

template <int NT>
__global__ __launch_bounds__(MX_THREADS)
void k_mx_down(int d, int I, int E, int budget, int ns, int nrec, int parts,
               const uint8_t *__restrict__ w2r, const uint8_t *__restrict__ w2s,
               const SpRec *__restrict__ rec, const float *__restrict__ pair_gate,
               const uint16_t *__restrict__ H, float *__restrict__ pairbuf) {
  __shared__ __attribute__((aligned(16))) uint8_t ring[MX_RING * NT * 4096];
  const MxWork k = mx_work(budget, ns, nrec, parts != 0, d / 16 / (MX_WAVES * MX_T), rec);
  if (k.n <= 0) return;
  const size_t eb = (size_t)(d / 16) * mx_tile_bytes(I);
  const uint8_t *w2 = k.u < E ? w2r + (size_t)k.u * eb : w2s + (size_t)(k.u - E) * eb;
  for (int c = 0; c < k.n; c += 16 * NT) {
    const int n = min(k.n - c, 16 * NT), p0 = k.p0 + c;
    if (c > 0) wg_barrier();
    sp_tiles<NT>((n + 15) / 16, [&](auto N) {
      mx_down_part<decltype(N)::value>(ring, k, d, I, w2, H + (size_t)p0 * I, n, pair_gate + p0,
                                       pairbuf + (size_t)p0 * d);
    });
  }
}

// ----------------------------------------------------------------- launch --
namespace {
// workgroups of `recs` records with RG row groups each, the same on every die
dim3 mx_grid(int recs, int RG) { return dim3((unsigned)(N_XCD * recs * ((RG + N_XCD - 1) / N_XCD))); }
}  // namespace

hipError_t launch_mx_gateup(const void *x, int B, int d, int I, int E, int K, int budget, int slots,
                            int ns, const void *w13, const void *w13s, const SpRec *rec,
                            const int32_t *sptok, void *H, hipStream_t st) {
  const bool parts = mx_parts(B);
  const int nrec = mx_records(B, K, budget, ns);
#define BASE_MXG(N)                                                                               \
  launch_k(k_mx_gateup<N>, mx_grid(parts ? nrec : slots + ns, I / 16 / MX_WAVES), dim3(MX_THREADS), \
           0, st, d, I, E, budget, ns, nrec, (int)parts, B * (K + ns), (const uint8_t *)w13,      \
           (const uint8_t *)w13s, rec, sptok, (const uint16_t *)x, B, (uint16_t *)H)
  if (B <= 16) BASE_MXG(1);
  else if (B <= 32) BASE_MXG(2);
  else BASE_MXG(MX_NT);
#undef BASE_MXG
  return hipGetLastError();
}

hipError_t launch_mx_down(int B, int d, int I, int E, int K, int budget, int slots, int ns,
                          const void *w2, const void *w2s, const SpRec *rec, const float *pair_gate,
                          const void *H, float *pairbuf, hipStream_t st) {
  const bool parts = mx_parts(B);
  const int nrec = mx_records(B, K, budget, ns);
#define BASE_MXD(N)                                                                                \
  launch_k(k_mx_down<N>, mx_grid(parts ? nrec : slots + ns, d / 16 / (MX_WAVES * MX_T)),           \
           dim3(MX_THREADS), 0, st, d, I, E, budget, ns, nrec, (int)parts, (const uint8_t *)w2,    \
           (const uint8_t *)w2s, rec, pair_gate, (const uint16_t *)H, pairbuf)
  if (B <= 16) BASE_MXD(1);
  else if (B <= 32) BASE_MXD(2);
  else BASE_MXD(MX_NT);
#undef BASE_MXD
  return hipGetLastError();
}

}  // namespace basek
