// Microscaled 4-bit floating point: rows quantised and read back, and the
// expert weights' packed layout (BASE_W_MXFP4).
//
// A block is 32 consecutive elements of a row, its scale 2^(s - 127) with the
// byte s = max(floor(log2 of the block's largest magnitude) + 125, 0), so that
// the largest element falls into [4, 8) where E2M1's largest value is 6; an
// element's code is v / scale rounded to the nearest E2M1 value, ties to the
// even code, beyond 6 to 6.  A block holding NaN or an infinity has s = 255 (the
// scale format's NaN) and codes 0; a block of zeros s = 0.  The exponent is read
// from the largest magnitude's bits: the comparison of magnitudes as integers
// puts infinities and NaN on top, so the same maximum finds them.
//
// The conversions are the gfx950 scale-converts (v_cvt_scalef32_*_fp4), whose
// scale operand is the float with the byte as its exponent field (0: 2^-127,
// 255: NaN); checked over every code and scale byte.  These kernels are streams:
// 16 bytes in or out per lane and access.  A Qwen3-shaped layer's gate and up
// weights (196,608 rows of 2048 bf16, 1.02 GB moved) take 214 us to quantise (4.8
// TB/s) and 160 to read back (6.4 TB/s), one expert's 3.8 us either way, of which
// its 8 MB are 1.6 and the rest is the launch and the first loads.
#include "common.hpp"
#include "internal.hpp"
#include "mx.hpp"

namespace basek {

constexpr int MXQ_THREADS = 256;
constexpr int MXQ_ROWS = 4;   // row sets per workgroup, their loads in flight together
constexpr long long MXQ_BLOCKS = 1 << 22;   // workgroups at most; they stride over the rows

// Eight consecutive elements of a row, as fp32.  VEC: 16-byte loads.
template <bool VEC>
__device__ __forceinline__ void mx_load8(const uint16_t *p, float (&v)[8]) {
  if (VEC) {
    const u32x4 q = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(q[i] << 16);
      v[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf16_to_f32(p[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void mx_load8(const float *p, float (&v)[8]) {
  if (VEC) {
    const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
  }
}

__device__ __forceinline__ uint32_t mx_mag(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
// the scale byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t mx_byte(uint32_t top) {
  const int e = (int)(top >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
// eight elements' codes, element i in bits 4 i
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8], uint32_t byte) {
  const float sc = mx_scale(byte);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], sc, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], sc, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], sc, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], sc, 3);
  return byte == 255u ? 0u : r;
}

// The rows of a workgroup: `tpr` threads a row (eight elements each at a
// time), `rps` rows at once, MXQ_ROWS sets of them.
struct MxqPlace {
  int r, c;   // row in a set (rps or more: none), first element
};
__device__ __forceinline__ MxqPlace mxq_place(int tpr, int rps) {
  const int t = threadIdx.x, r = t / tpr;
  return {r < rps ? r : rps, 8 * (t - r * tpr)};
}

// Four lanes a block: the quad's largest magnitude by two quad permutations.
template <typename T, bool VEC>
__global__ __launch_bounds__(MXQ_THREADS)
void k_mx_quantize(const T *__restrict__ src, long long rows, int cols, long long ld, int tpr,
                   int rps, uint32_t *__restrict__ codes, uint8_t *__restrict__ scales) {
  const MxqPlace pl = mxq_place(tpr, rps);
  if (pl.r >= rps) return;   // whole quads: tpr is a multiple of four
  const long long set = rps * MXQ_ROWS;
  for (long long r0 = blockIdx.x * set + pl.r; r0 < rows; r0 += gridDim.x * set)
  for (int c = pl.c; c < cols; c += 8 * tpr) {
    float v[MXQ_ROWS][8];
#pragma unroll
    for (int i = 0; i < MXQ_ROWS; ++i) {
      const long long r = r0 + i * rps;
      if (r < rows) mx_load8<VEC>(src + r * ld + c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < MXQ_ROWS; ++i) {
      const long long r = r0 + i * rps;
      if (r >= rows) break;
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < 8; ++q) m = max(m, mx_mag(v[i][q]));
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));
      const uint32_t byte = mx_byte(m);
      codes[(r * cols + c) >> 3] = mx_encode8(v[i], byte);
      if ((threadIdx.x & 3) == 0) scales[(r * cols + c) >> 5] = (uint8_t)byte;
    }
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(MXQ_THREADS)
void k_mx_dequantize(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                     long long rows, int cols, int tpr, int rps, T *__restrict__ dst,
                     long long ld) {
  const MxqPlace pl = mxq_place(tpr, rps);
  if (pl.r >= rps) return;
  const long long set = rps * MXQ_ROWS;
  for (long long r0 = blockIdx.x * set + pl.r; r0 < rows; r0 += gridDim.x * set)
  for (int c = pl.c; c < cols; c += 8 * tpr) {
    uint32_t q[MXQ_ROWS], s[MXQ_ROWS];
#pragma unroll
    for (int i = 0; i < MXQ_ROWS; ++i) {
      const long long r = r0 + i * rps;
      if (r < rows) {
        q[i] = codes[(r * cols + c) >> 3];
        s[i] = scales[(r * cols + c) >> 5];
      }
    }
#pragma unroll
    for (int i = 0; i < MXQ_ROWS; ++i) {
      const long long r = r0 + i * rps;
      if (r >= rows) break;
      T *o = dst + r * ld + c;
      const float sc = mx_scale(s[i]);
      if constexpr (sizeof(T) == 2) {
        const u32x4 w = __builtin_bit_cast(u32x4, mx_decode8(q[i], sc));
        if (VEC) {
          *reinterpret_cast<u32x4 *>(o) = w;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
        }
      } else {
        float w[8];
        mx_decode8_f32(q[i], sc, w);
        if (VEC) {
          reinterpret_cast<f32x4 *>(o)[0] = f32x4{w[0], w[1], w[2], w[3]};
          reinterpret_cast<f32x4 *>(o)[1] = f32x4{w[4], w[5], w[6], w[7]};
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = w[e];
        }
      }
    }
  }
}

// ---------------------------------------------------------------- experts --
// One workgroup per chunk of a 16-row tile (four steps of 128 elements, one
// per wavefront): a lane's 16 bytes of a step are one block of one row.
// Source row of tile t: w13 (t even: gate, odd: up) I (t & 1) + 16 (t / 2),
// w2 16 t, plus lane % 16.
struct MxTilePos {
  size_t row;    // this lane's source row
  int k;         // its block's first element in this wavefront's step
  uint8_t *dst;  // the chunk
};
__device__ __forceinline__ MxTilePos mx_tile_pos(uint8_t *out, int K, int tiles, int rows_per_e,
                                                 int I, int gate_up) {
  const int lane = lane_id(), C = mx_chunks(K);
  const int c = (int)(blockIdx.x % (unsigned)C), t = (int)(blockIdx.x / (unsigned)C);
  const size_t u = blockIdx.y;
  const int row = (gate_up ? (t & 1) * I + 16 * (t >> 1) : 16 * t) + (lane & 15);
  return {u * rows_per_e + row, MX_STEP * (MX_CHUNK * c + wave_id()) + 32 * (lane >> 4),
          out + (u * tiles + t) * mx_tile_bytes(K) + (size_t)c * MX_CHUNK_BYTES};
}
// the wavefront's step of the chunk, and, once all four are known, the
// chunk's scales (byte j of lane l: its block's in step j)
__device__ __forceinline__ void mx_put(const MxTilePos &p, int K, u32x4 codes, uint32_t byte) {
  __shared__ uint8_t sc[MX_CHUNK * WAVE];
  const int lane = lane_id(), w = wave_id();
  if (p.k - 32 * (lane >> 4) < K)   // steps past the row do not exist
    *reinterpret_cast<u32x4 *>(p.dst + 256 + w * 1024 + lane * 16) = codes;
  sc[lane * 4 + w] = (uint8_t)byte;
  __syncthreads();
  if (w == 0)
    *reinterpret_cast<uint32_t *>(p.dst + lane * 4) = reinterpret_cast<const uint32_t *>(sc)[lane];
}

__global__ __launch_bounds__(MX_CHUNK * WAVE)
void k_mx_pack(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int K,
               int tiles, int rows_per_e, int I, int gate_up, uint8_t *__restrict__ out) {
  const MxTilePos p = mx_tile_pos(out, K, tiles, rows_per_e, I, gate_up);
  u32x4 v = {0, 0, 0, 0};
  uint32_t byte = 0;
  if (p.k < K) {
    v = *reinterpret_cast<const u32x4 *>(codes + p.row * (size_t)(K / 2) + p.k / 2);
    byte = scales[p.row * (size_t)(K / 32) + p.k / 32];
  }
  mx_put(p, K, v, byte);
}

template <typename T>
__global__ __launch_bounds__(MX_CHUNK * WAVE)
void k_mx_quantize_experts(const T *__restrict__ w, int K, int tiles, int rows_per_e, int I,
                           int gate_up, uint8_t *__restrict__ out) {
  const MxTilePos p = mx_tile_pos(out, K, tiles, rows_per_e, I, gate_up);
  u32x4 codes = {0, 0, 0, 0};
  uint32_t byte = 0;
  if (p.k < K) {
    float v[4][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mx_load8<true>(w + p.row * (size_t)K + p.k + 8 * i, v[i]);
#pragma unroll
      for (int q = 0; q < 8; ++q) m = max(m, mx_mag(v[i][q]));
    }
    byte = mx_byte(m);
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = mx_encode8(v[i], byte);
  }
  mx_put(p, K, codes, byte);
}

// ----------------------------------------------------------------- launch --
namespace {
struct MxqGrid {
  int tpr, rps;
  unsigned blocks;
};
MxqGrid mxq_grid(long long rows, int cols) {
  const int per_row = cols / 8;
  MxqGrid g;
  g.tpr = per_row < MXQ_THREADS ? per_row : MXQ_THREADS;
  g.rps = MXQ_THREADS / g.tpr;
  const long long set = (long long)g.rps * MXQ_ROWS;
  const long long sets = (rows + set - 1) / set;
  g.blocks = (unsigned)(sets < MXQ_BLOCKS ? sets : MXQ_BLOCKS);
  return g;
}
}  // namespace

hipError_t launch_mx_quantize(bool bf16, const void *src, long long rows, int cols, long long ld,
                              void *codes, uint8_t *scales, hipStream_t st) {
  const MxqGrid g = mxq_grid(rows, cols);
  const bool vec = (uintptr_t)src % 16 == 0 && ld % (bf16 ? 8 : 4) == 0;
#define BASE_MXQ(T, V)                                                                          \
  launch_k(k_mx_quantize<T, V>, dim3(g.blocks), dim3(MXQ_THREADS), 0, st, (const T *)src, rows, \
           cols, ld, g.tpr, g.rps, (uint32_t *)codes, scales)
  if (bf16) { if (vec) BASE_MXQ(uint16_t, true); else BASE_MXQ(uint16_t, false); }
  else { if (vec) BASE_MXQ(float, true); else BASE_MXQ(float, false); }
#undef BASE_MXQ
  return hipGetLastError();
}

hipError_t launch_mx_dequantize(bool bf16, const void *codes, const uint8_t *scales, long long rows,
                                int cols, void *dst, long long ld, hipStream_t st) {
  const MxqGrid g = mxq_grid(rows, cols);
  const bool vec = (uintptr_t)dst % 16 == 0 && ld % (bf16 ? 8 : 4) == 0;
#define BASE_MXD(T, V)                                                                      \
  launch_k(k_mx_dequantize<T, V>, dim3(g.blocks), dim3(MXQ_THREADS), 0, st,                 \
           (const uint32_t *)codes, scales, rows, cols, g.tpr, g.rps, (T *)dst, ld)
  if (bf16) { if (vec) BASE_MXD(uint16_t, true); else BASE_MXD(uint16_t, false); }
  else { if (vec) BASE_MXD(float, true); else BASE_MXD(float, false); }
#undef BASE_MXD
  return hipGetLastError();
}

hipError_t launch_mx_pack(const uint8_t *w13c, const uint8_t *w13s, const uint8_t *w2c,
                          const uint8_t *w2s, int E, int d, int I, void *w13, void *w2,
                          hipStream_t st) {
  launch_k(k_mx_pack, dim3((unsigned)(I / 8 * mx_chunks(d)), E), dim3(MX_CHUNK * WAVE), 0, st,
           w13c, w13s, d, I / 8, 2 * I, I, 1, (uint8_t *)w13);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  launch_k(k_mx_pack, dim3((unsigned)(d / 16 * mx_chunks(I)), E), dim3(MX_CHUNK * WAVE), 0, st,
           w2c, w2s, I, d / 16, d, I, 0, (uint8_t *)w2);
  return hipGetLastError();
}

hipError_t launch_mx_quantize_experts(bool bf16, const void *w13, const void *w2, int E, int d,
                                      int I, void *w13m, void *w2m, hipStream_t st) {
#define BASE_MXE(T, W, K, TILES, ROWS, GU, OUT)                                               \
  launch_k(k_mx_quantize_experts<T>, dim3((unsigned)((TILES) * mx_chunks(K)), E),            \
           dim3(MX_CHUNK * WAVE), 0, st, (const T *)W, K, TILES, ROWS, I, GU, (uint8_t *)OUT)
  if (bf16) BASE_MXE(uint16_t, w13, d, I / 8, 2 * I, 1, w13m);
  else BASE_MXE(float, w13, d, I / 8, 2 * I, 1, w13m);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (bf16) BASE_MXE(uint16_t, w2, I, d / 16, d, 0, w2m);
  else BASE_MXE(float, w2, I, d / 16, d, 0, w2m);
#undef BASE_MXE
  return hipGetLastError();
}

}  // namespace basek
