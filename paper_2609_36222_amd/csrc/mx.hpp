// The packed layout of 4-bit expert weights (BASE_W_MXFP4) and the conversions.
//
// A matrix is cut into 16-row tiles; w13's are ordered gate tile r, up tile r,
// gate tile r + 1, ..  A tile holds its contraction of K elements as steps of
// 128, grouped in chunks of four: first the chunk's scales, 64 lanes x 4 bytes
// (byte j: the scale of the lane's block in the chunk's step j), then its steps,
// 64 lanes x 16 bytes each, lane l holding row l % 16, block l / 16 of the step
// (elements 32 (l / 16) .. +31, the low half byte first).  The last chunk holds
// only the steps there are; blocks past K (K / 64 odd) are zeros.
//
// Why: a lane's 16 bytes are four MFMA operands with one scale, so a step of a
// tile costs one load and one scale byte per lane and no byte is read twice (a
// layout in the instruction's own element order needs each scale in four lanes,
// or 8-byte loads).  The contraction's order inside a step is free as long as
// both operands agree: operand f (0 .. 3) takes the elements 8 f .. 8 f + 7 of
// every block, so the token side gives lane (token, g) the elements 32 g + 8 f ..
#pragma once

#include "common.hpp"

namespace basek {

constexpr int MX_STEP = 128;    // contraction elements per step
constexpr int MX_CHUNK = 4;     // steps per chunk
constexpr int MX_CHUNK_BYTES = 256 + MX_CHUNK * 1024;

__host__ __device__ inline int mx_steps(int K) { return (K + MX_STEP - 1) / MX_STEP; }
__host__ __device__ inline int mx_chunks(int K) { return (mx_steps(K) + MX_CHUNK - 1) / MX_CHUNK; }
__host__ __device__ inline size_t mx_tile_bytes(int K) {
  return (size_t)mx_chunks(K) * 256 + (size_t)mx_steps(K) * 1024;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// a scale byte as the converts' scale operand
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight codes (the low half byte first) to bf16, exactly (values below bf16's
// smallest normal included)
__device__ __forceinline__ bf16x8 mx_decode8(uint32_t q, float sc) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc, 3);
  return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                          __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}
__device__ __forceinline__ void mx_decode8_f32(uint32_t q, float sc, float (&v)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, sc, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, sc, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, sc, 2);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, sc, 3);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
  v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}

}  // namespace basek
