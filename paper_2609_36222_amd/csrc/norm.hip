// RMS norms around a block, fused with its gate and the residual scale:
//   h' = a h + g * (w_post n(y))       (y itself without a post gain)
//   x' = w_pre n(h')                   n(v) = v / sqrt(mean v^2 + eps)
// over rows of d elements, everything in fp32 and each output rounded once (x'
// from h' before its rounding, so that the next block's input does not carry the
// residual stream's).  A row whose mean v^2 + eps is 0 has n(v) = 0.
//
// Bound by memory: y and h are read once, h' and x' written once, and the row
// lives in registers between the two means, TPR threads with EPT elements each.
// One wavefront a row up to 1024 elements (no barrier, several rows per
// workgroup), beyond it one workgroup, whose wavefronts join their sums through
// LDS.
#include "common.hpp"
#include "internal.hpp"

namespace basek {

struct NormArgs {
  int d;
  float eps, scale;
  const float *post, *gate, *pre;
  long long gate_ld;
};

template <typename T> struct Vec16;
template <> struct Vec16<float> { static constexpr int N = 4; };
template <> struct Vec16<uint16_t> { static constexpr int N = 8; };

__device__ __forceinline__ float norm_get(const float *p) { return *p; }
__device__ __forceinline__ float norm_get(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void norm_put(float *p, float v) { *p = v; }
__device__ __forceinline__ void norm_put(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// V consecutive elements (V = 1, or 16 bytes of T, of fp32 in pieces of four)
template <int V, typename T>
__device__ __forceinline__ void norm_load(const T *p, float *v) {
  if constexpr (V == 1) {
    v[0] = norm_get(p);
  } else if constexpr (sizeof(T) == 2) {
    const u32x4 q = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(q[i] << 16);
      v[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 q = *reinterpret_cast<const f32x4 *>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = q[e];
    }
  }
}
template <int V, typename T>
__device__ __forceinline__ void norm_store(T *p, const float *v) {
  if constexpr (V == 1) {
    norm_put(p, v[0]);
  } else if constexpr (sizeof(T) == 2) {
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
    *reinterpret_cast<u32x4 *>(p) = q;
  } else {
    *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
  }
}

// Sum over the row's threads, the same value in all of them: a butterfly in
// the wavefront, then (TPR > 64) the wavefronts' sums in ascending order.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red) {
  v = wave_tree_sum(v);
  if constexpr (TPR > WAVE) {
    if (lane_id() == 0) red[wave_id()] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / WAVE; ++i) v = v + red[i];
  }
  return v;
}

// 1 / sqrt(mean + eps), 0 for a row of nothing
__device__ __forceinline__ float row_rstd(float sum, int d, float eps) {
  const float m = sum / (float)d + eps;
  return m > 0.0f ? 1.0f / __fsqrt_rn(m) : (m == 0.0f ? 0.0f : m);   // NaN stays NaN
}

// One row.  Element i V + e of this thread's EPT is column (i TPR + tid) V + e; ly
// loads V of y's (HAS_Y: there is a block's output), h its residual stream.
template <typename T, int TPR, int EPT, int V, bool HAS_Y, typename LY>
__device__ __forceinline__ void norm_row(const NormArgs &a, long long row, int tid, LY ly, const T *h,
                                         T *ho, T *xo, float *red) {
  float v[EPT], s[EPT];
  const int d = a.d;
  constexpr int Q = EPT / V;
#define BASE_EACH(i, c)                                    \
  _Pragma("unroll") for (int i = 0; i < Q; ++i)            \
    if (const int c = (i * TPR + tid) * V; c < d)
#pragma unroll
  for (int i = 0; i < EPT; ++i) v[i] = s[i] = 0.0f;
  BASE_EACH(i, c) norm_load<V>(h + c, &v[i * V]);
  if (HAS_Y) {
    BASE_EACH(i, c) ly(c, &s[i * V]);
    float r = 1.0f;
    if (a.post) {
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) ss = __builtin_fmaf(s[i], s[i], ss);
      r = row_rstd(row_sum<TPR>(ss, red), d, a.eps);
    }
    BASE_EACH(i, c) {
      float w[V], g[V];
      if (a.post) norm_load<V>(a.post + c, w);
      if (a.gate) norm_load<V>(a.gate + row * a.gate_ld + c, g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float t = s[i * V + e];
        if (a.post) t = t * r * w[e];
        if (a.gate) t = t * g[e];
        v[i * V + e] = __builtin_fmaf(a.scale, v[i * V + e], t);
      }
    }
    if (ho) BASE_EACH(i, c) norm_store<V>(ho + c, &v[i * V]);
  }
  if (xo) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
    const float r = row_rstd(row_sum<TPR>(ss, red + 16), d, a.eps);
    BASE_EACH(i, c) {
      float w[V];
      norm_load<V>(a.pre + c, w);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i * V + e] = v[i * V + e] * r * w[e];
      norm_store<V>(xo + c, &v[i * V]);
    }
  }
#undef BASE_EACH
}

// RPW rows per workgroup (TPR = 64: one per wavefront).  ho may be h and xo may
// be y: a thread's elements are read before it writes them.
template <typename T, int TPR, int EPT, int V, int RPW, bool HAS_Y>
__global__ __launch_bounds__(TPR * RPW)
void k_norm(NormArgs a, long long rows, const T *y, long long y_ld, const T *h, long long h_ld,
            T *ho, long long ho_ld, T *xo, long long xo_ld) {
  __shared__ float red[TPR > WAVE ? 32 : 1];
  for (long long row = (long long)blockIdx.x * RPW + (RPW > 1 ? wave_id_u() : 0); row < rows;
       row += (long long)gridDim.x * RPW) {
    const T *yr = y + (HAS_Y ? row * y_ld : 0);
    norm_row<T, TPR, EPT, V, HAS_Y>(a, row, RPW > 1 ? lane_id() : (int)threadIdx.x,
                                    [&](int c, float *s) { norm_load<V>(yr + c, s); },
                                    h + row * h_ld, ho ? ho + row * ho_ld : nullptr,
                                    xo ? xo + row * xo_ld : nullptr, red);
    if (TPR > WAVE) __syncthreads();   // red is free for the next row
  }
}

// The layer's combine and the norm behind it: y_t = sum_j pairbuf[pair_of[t][j]]
// in j order, rounded to T as base_decode_layer writes it, then the row.
template <typename T, int TPR, int EPT, int V>
__global__ __launch_bounds__(TPR)
void k_combine_norm(NormArgs a, int kc, const int32_t *__restrict__ pair_of,
                    const float *__restrict__ pairbuf, const T *h, T *ho, T *xo) {
  __shared__ float red[32];
  __shared__ int pair_s[MAX_K + MAX_SHARED];
  const int t = blockIdx.x, d = a.d;
  if ((int)threadIdx.x < kc) pair_s[threadIdx.x] = pair_of[(size_t)t * kc + threadIdx.x];
  __syncthreads();
  norm_row<T, TPR, EPT, V, true>(
      a, t, threadIdx.x,
      [&](int c, float *s) {
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        for (int j = 0; j < kc; ++j) {
          const int p = pair_s[j];
          if (p < 0) continue;   // a routed rank the token does not execute
          float v[V];
          norm_load<V>(pairbuf + (size_t)p * d + c, v);
#pragma unroll
          for (int e = 0; e < V; ++e) acc[e] = acc[e] + v[e];
        }
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = sizeof(T) == 2 ? bf16_to_f32(f32_to_bf16(acc[e])) : acc[e];
      },
      h + (size_t)t * d, ho ? ho + (size_t)t * d : nullptr, xo ? xo + (size_t)t * d : nullptr, red);
}

// The shapes of a row by its length, LAUNCH(threads a row, elements a thread, rows a
// workgroup).  k_norm and k_combine_norm take the same ones, so that their sums
// have the same order and the block call the bits of its parts.
#define BASE_NORM_SHAPES(d, LAUNCH)       \
  do {                                    \
    if ((d) <= 512) LAUNCH(64, 8, 4);     \
    else if ((d) <= 1024) LAUNCH(64, 16, 4); \
    else if ((d) <= 2048) LAUNCH(256, 8, 1); \
    else if ((d) <= 4096) LAUNCH(256, 16, 1); \
    else if ((d) <= 8192) LAUNCH(512, 16, 1); \
    else LAUNCH(1024, 16, 1);             \
  } while (0)

namespace {
constexpr long long NORM_BLOCKS = 1 << 22;   // workgroups at most; they stride over the rows

template <typename T, int V>
hipError_t norm_launch(const NormArgs &a, long long rows, const void *y, long long y_ld,
                       const void *h, long long h_ld, void *ho, long long ho_ld, void *xo,
                       long long xo_ld, hipStream_t st) {
#define BASE_NORM(TPR, EPT, RPW)                                                              \
  do {                                                                                        \
    const long long b = (rows + (RPW)-1) / (RPW);                                             \
    const auto kern = y ? k_norm<T, TPR, EPT, V, RPW, true> : k_norm<T, TPR, EPT, V, RPW, false>; \
    launch_k(kern, dim3((unsigned)(b < NORM_BLOCKS ? b : NORM_BLOCKS)), dim3((TPR) * (RPW)),  \
             0, st, a, rows, (const T *)y, y_ld, (const T *)h, h_ld, (T *)ho, ho_ld, (T *)xo, \
             xo_ld);                                                                          \
  } while (0)
  BASE_NORM_SHAPES(a.d, BASE_NORM);
#undef BASE_NORM
  return hipGetLastError();
}
}  // namespace

hipError_t launch_norm(bool bf16, int d, float eps, float scale, const float *post, const float *gate,
                       long long gate_ld, const float *pre, long long rows, const void *y,
                       long long y_ld, const void *h, long long h_ld, void *ho, long long ho_ld,
                       void *xo, long long xo_ld, hipStream_t st) {
  const NormArgs a{d, eps, scale, post, gate, pre, gate_ld};
  const int n = bf16 ? 8 : 4;
  // 16-byte accesses: whole vectors in every row, and rows and gains that start on 16 bytes
  auto ok = [](const void *p, long long ld, int n) {
    return !p || ((uintptr_t)p % 16 == 0 && ld % n == 0);
  };
  const bool vec = d % n == 0 && ok(y, y_ld, n) && ok(h, h_ld, n) && ok(ho, ho_ld, n) &&
                   ok(xo, xo_ld, n) && ok(post, 0, 4) && ok(gate, gate_ld, 4) && ok(pre, 0, 4);
#define BASE_NL(T, V) norm_launch<T, V>(a, rows, y, y_ld, h, h_ld, ho, ho_ld, xo, xo_ld, st)
  if (bf16) return vec ? BASE_NL(uint16_t, 8) : BASE_NL(uint16_t, 1);
  return vec ? BASE_NL(float, 4) : BASE_NL(float, 1);
#undef BASE_NL
}

hipError_t launch_combine_norm(bool bf16, int B, int d, int kc, const int32_t *pair_of,
                               const float *pairbuf, float eps, float scale, const float *post,
                               const float *gate, long long gate_ld, const float *pre, const void *h,
                               void *ho, void *xo, hipStream_t st) {
  const NormArgs a{d, eps, scale, post, gate, pre, gate_ld};
#define BASE_CN(TPR, EPT, RPW)                                                                  \
  do {                                                                                          \
    if (bf16)                                                                                   \
      launch_k(k_combine_norm<uint16_t, TPR, EPT, 8>, dim3(B), dim3(TPR), 0, st, a, kc, pair_of, \
               pairbuf, (const uint16_t *)h, (uint16_t *)ho, (uint16_t *)xo);                   \
    else                                                                                        \
      launch_k(k_combine_norm<float, TPR, EPT, 4>, dim3(B), dim3(TPR), 0, st, a, kc, pair_of,   \
               pairbuf, (const float *)h, (float *)ho, (float *)xo);                            \
  } while (0)
  BASE_NORM_SHAPES(d, BASE_CN);
#undef BASE_CN
  return hipGetLastError();
}

}  // namespace basek
