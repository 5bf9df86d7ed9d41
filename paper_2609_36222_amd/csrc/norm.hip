// RMS norms around a block, fused with its gate and the residual scale:
//   h' = a h + g * (w_post n(y))       (y itself without a post gain)
//   x' = w_pre n(h')                   n(v) = v / sqrt(mean v^2 + eps)
// over rows of d elements, everything in fp32 and each output rounded once (x'
// from h' before its rounding, so that the next block's input does not carry the
// residual stream's).  A row whose mean v^2 + eps is 0 has n(v) = 0.
//
// Bound by memory: y and h are read once, h' and x' written once, and the row
// lives in registers between the two means, EPT elements a thread.  A row of up to
// 1024 elements is one wavefront's (no barrier, four rows a workgroup), a longer
// one a workgroup's, whose wavefronts join their sums through LDS; the threads
// follow from d (norm_threads).  A workgroup takes rows in turn, so that the
// gains, read once, stay in registers.  Accesses are 16 bytes at any element
// alignment: rows of odd length start anywhere, and global loads need no more
// than element alignment; a row's last piece, if it is not whole, goes by
// elements.  8191 rows of 5001 fp32 elements: 129 us, 5.1 TB/s, the rate of a large
// copy; with element accesses 226.  One row of 2048: 3.2 us, its two reductions and
// the launch; 255 rows of 4096 6.0 us.
#include "common.hpp"
#include "internal.hpp"

namespace basek {

struct NormArgs {
  int d;
  float eps, scale;
  const float *post, *gate, *pre;
  long long gate_ld;
};

// 16 bytes at the alignment of T
struct __attribute__((packed, aligned(4))) Any16F { f32x4 v; };
struct __attribute__((packed, aligned(2))) Any16H { u32x4 v; };

__device__ __forceinline__ float norm_get(const float *p) { return *p; }
__device__ __forceinline__ float norm_get(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void norm_put(float *p, float v) { *p = v; }
__device__ __forceinline__ void norm_put(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// V (4 or 8) consecutive elements, `left` of them in the row (zeros past it)
template <int V>
__device__ __forceinline__ void norm_load(const float *p, int left, float *v) {
  if (left >= V) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 q = reinterpret_cast<const Any16F *>(p + i)->v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = q[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < left ? p[e] : 0.0f;
  }
}
template <int V>
__device__ __forceinline__ void norm_load(const uint16_t *p, int left, float *v) {
  static_assert(V == 8, "16 bytes of bf16");
  if (left >= V) {
    const u32x4 q = reinterpret_cast<const Any16H *>(p)->v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(q[i] << 16);
      v[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < left ? bf16_to_f32(p[e]) : 0.0f;
  }
}
template <int V>
__device__ __forceinline__ void norm_store(float *p, int left, const float *v) {
  if (left >= V) {
    reinterpret_cast<Any16F *>(p)->v = f32x4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < left) p[e] = v[e];
  }
}
template <int V>
__device__ __forceinline__ void norm_store(uint16_t *p, int left, const float *v) {
  if (left >= V) {
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
    reinterpret_cast<Any16H *>(p)->v = q;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < left) p[e] = f32_to_bf16(v[e]);
  }
}

// Elements a thread and threads a row: the same for k_norm and k_combine_norm, so
// that their sums have one order and the block call the bits of its parts.
__host__ __device__ inline int norm_ept(int d) { return d <= 512 || (d > 1024 && d <= 2048) ? 8 : 16; }
__host__ __device__ inline int norm_threads(int d) {
  const int per = WAVE * norm_ept(d);
  return (d + per - 1) / per * WAVE;
}
static_assert(MAX_NORM_D <= 16 * 1024, "a row in one workgroup's registers");

// Sum over the row's threads, the same value in all of them: a butterfly in
// the wavefront, then (WG: the row is a workgroup's) the wavefronts' sums in
// ascending order.
template <bool WG>
__device__ __forceinline__ float row_sum(float v, float *red) {
  v = wave_tree_sum(v);
  if constexpr (WG) {
    const int nw = (int)blockDim.x / WAVE;
    if (lane_id() == 0) red[wave_id()] = v;
    __syncthreads();
    v = red[0];
    for (int i = 1; i < nw; ++i) v = v + red[i];
  }
  return v;
}

// 1 / sqrt(mean + eps), 0 for a row of nothing
__device__ __forceinline__ float row_rstd(float sum, int d, float eps) {
  const float m = sum / (float)d + eps;
  return m > 0.0f ? 1.0f / __fsqrt_rn(m) : (m == 0.0f ? 0.0f : m);   // NaN stays NaN
}

// A thread's share of rows: piece i of V elements starts at column (i threads + tid) V.
template <typename T, int EPT, bool WG>
struct NormRow {
  static constexpr int V = 16 / sizeof(T), Q = EPT / V;
  float post[EPT], pre[EPT], gate[EPT];
  int tid, threads;
  __device__ int col(int i) const { return (i * threads + tid) * V; }
  template <typename P>
  __device__ void load(const P *p, int d, float (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) norm_load<V>(p + col(i), d - col(i), &v[i * V]);
  }
  // the parameters that every row shares
  __device__ void params(const NormArgs &a, bool pre_needed) {
    if (a.post) load(a.post, a.d, post);
    if (a.gate && a.gate_ld == 0) load(a.gate, a.d, gate);
    if (pre_needed) load(a.pre, a.d, pre);
  }
  // one row from h (v) and, with HAS_Y, the block's output (s)
  template <bool HAS_Y>
  __device__ void run(const NormArgs &a, float (&v)[EPT], float (&s)[EPT], T *ho, T *xo, float *red) {
    const int d = a.d;
    if (HAS_Y) {
      float r = 1.0f;
      if (a.post) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < EPT; ++i) ss = __builtin_fmaf(s[i], s[i], ss);
        r = row_rstd(row_sum<WG>(ss, red), d, a.eps);
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        float t = s[i];
        if (a.post) t = t * r * post[i];
        if (a.gate) t = t * gate[i];
        v[i] = __builtin_fmaf(a.scale, v[i], t);
      }
      if (ho) {
#pragma unroll
        for (int i = 0; i < Q; ++i) norm_store<V>(ho + col(i), d - col(i), &v[i * V]);
      }
    }
    if (xo) {
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
      const float r = row_rstd(row_sum<WG>(ss, red + 16), d, a.eps);
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] = v[i] * r * pre[i];
#pragma unroll
      for (int i = 0; i < Q; ++i) norm_store<V>(xo + col(i), d - col(i), &v[i * V]);
    }
  }
};

// ho may be h or y and xo may be y or h: a thread's elements are read before it
// writes them.
template <typename T, int EPT, bool WG, bool HAS_Y>
__global__ __launch_bounds__(WG ? 1024 : 256)
void k_norm(NormArgs a, long long rows, const T *y, long long y_ld, const T *h, long long h_ld,
            T *ho, long long ho_ld, T *xo, long long xo_ld) {
  __shared__ float red[WG ? 32 : 1];
  NormRow<T, EPT, WG> n;
  n.tid = WG ? (int)threadIdx.x : lane_id();
  n.threads = WG ? (int)blockDim.x : WAVE;
  const int per = WG ? 1 : (int)blockDim.x / WAVE;
  bool first = true;
  for (long long row = (long long)blockIdx.x * per + (WG ? 0 : wave_id_u()); row < rows;
       row += (long long)gridDim.x * per) {
    float v[EPT], s[EPT];
    n.load(h + row * h_ld, a.d, v);
    if (HAS_Y) {
      n.load(y + row * y_ld, a.d, s);
      if (a.gate && a.gate_ld != 0) n.load(a.gate + row * a.gate_ld, a.d, n.gate);
    }
    if (first) n.params(a, xo != nullptr);
    first = false;
    n.template run<HAS_Y>(a, v, s, ho ? ho + row * ho_ld : nullptr, xo ? xo + row * xo_ld : nullptr, red);
    if (WG) __syncthreads();   // red is free for the next row
  }
}

// The layer's combine and the norm behind it: y_t = sum_j pairbuf[pair_of[t][j]]
// in j order, rounded to T as base_decode_layer writes it, then the row.
// SPLIT: a pair's row is the sum of `shares` rows `stride` apart, in their order.
template <typename T, int EPT, bool WG, bool SPLIT>
__global__ __launch_bounds__(WG ? 1024 : WAVE)
void k_combine_norm(NormArgs a, int kc, const int32_t *__restrict__ pair_of,
                    const float *__restrict__ pairbuf, int shares, size_t stride, const T *h, T *ho,
                    T *xo) {
  __shared__ float red[WG ? 32 : 1];
  constexpr int GROUP = 4;   // ranks whose rows are in flight together
  NormRow<T, EPT, WG> n;
  n.tid = threadIdx.x;
  n.threads = blockDim.x;
  const size_t t = blockIdx.x;
  const int d = a.d;
  float v[EPT], s[EPT];
  n.load(h + t * d, d, v);
#pragma unroll
  for (int i = 0; i < EPT; ++i) s[i] = 0.0f;
  for (int j0 = 0; j0 < kc; j0 += GROUP) {
    int p[GROUP];
#pragma unroll
    for (int g = 0; g < GROUP; ++g) p[g] = j0 + g < kc ? pair_of[t * kc + j0 + g] : -1;
    // a rank without a pair reads row 0: with a branch around each load they do not
    // go out together (B = 16 and 64, d = 2048: 6.8 and 7.4 us against 5.8 and 5.9)
    float o[GROUP][EPT];
#pragma unroll
    for (int g = 0; g < GROUP; ++g) n.load(pairbuf + (size_t)max(p[g], 0) * d, d, o[g]);
#pragma unroll
    for (int g = 0; g < GROUP; ++g) {
      if (p[g] < 0) continue;   // a routed rank the token does not execute
      for (int q = 1; SPLIT && q < shares; ++q) {
        float e[EPT];
        n.load(pairbuf + q * stride + (size_t)p[g] * d, d, e);
#pragma unroll
        for (int i = 0; i < EPT; ++i) o[g][i] = o[g][i] + e[i];
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[i] = s[i] + o[g][i];
    }
  }
  if (a.gate && a.gate_ld != 0) n.load(a.gate + t * a.gate_ld, d, n.gate);
  n.params(a, xo != nullptr);
#pragma unroll
  for (int i = 0; i < EPT; ++i) s[i] = sizeof(T) == 2 ? bf16_to_f32(f32_to_bf16(s[i])) : s[i];
  n.template run<true>(a, v, s, ho ? ho + t * d : nullptr, xo ? xo + t * d : nullptr, red);
}

hipError_t launch_norm(bool bf16, int d, float eps, float scale, const float *post, const float *gate,
                       long long gate_ld, const float *pre, long long rows, const void *y,
                       long long y_ld, const void *h, long long h_ld, void *ho, long long ho_ld,
                       void *xo, long long xo_ld, int n_cu, hipStream_t st) {
  const NormArgs a{d, eps, scale, post, gate, pre, gate_ld};
  const bool wg = norm_threads(d) > WAVE;
  const int threads = wg ? norm_threads(d) : 4 * WAVE, per = wg ? 1 : 4;
  // sixteen wavefronts a CU, in workgroups that stride over the rows
  const long long most = (long long)n_cu * (16 * WAVE / threads > 0 ? 16 * WAVE / threads : 1);
  const long long blocks = (rows + per - 1) / per;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
#define BASE_NORM(T, EPT, WG)                                                                    \
  launch_k(y ? k_norm<T, EPT, WG, true> : k_norm<T, EPT, WG, false>, grid, dim3(threads), 0, st, \
           a, rows, (const T *)y, y_ld, (const T *)h, h_ld, (T *)ho, ho_ld, (T *)xo, xo_ld)
#define BASE_NORM_T(T)                                                                           \
  do {                                                                                           \
    if (wg) { if (norm_ept(d) == 8) BASE_NORM(T, 8, true); else BASE_NORM(T, 16, true); }        \
    else { if (norm_ept(d) == 8) BASE_NORM(T, 8, false); else BASE_NORM(T, 16, false); }         \
  } while (0)
  if (bf16) BASE_NORM_T(uint16_t);
  else BASE_NORM_T(float);
#undef BASE_NORM_T
#undef BASE_NORM
  return hipGetLastError();
}

hipError_t launch_combine_norm(bool bf16, int B, int d, int kc, const int32_t *pair_of,
                               const float *pairbuf, int shares, size_t stride, float eps,
                               float scale, const float *post, const float *gate,
                               long long gate_ld, const float *pre, const void *h, void *ho,
                               void *xo, hipStream_t st) {
  const NormArgs a{d, eps, scale, post, gate, pre, gate_ld};
  const int threads = norm_threads(d);
#define BASE_CN(T, EPT, WG)                                                                      \
  launch_k(shares > 1 ? k_combine_norm<T, EPT, WG, sizeof(T) == 2>                               \
                      : k_combine_norm<T, EPT, WG, false>,                                       \
           dim3(B), dim3(threads), 0, st, a, kc, pair_of, pairbuf, shares, stride, (const T *)h, \
           (T *)ho, (T *)xo)
#define BASE_CN_T(T)                                                                             \
  do {                                                                                           \
    if (threads > WAVE) { if (norm_ept(d) == 8) BASE_CN(T, 8, true); else BASE_CN(T, 16, true); } \
    else { if (norm_ept(d) == 8) BASE_CN(T, 8, false); else BASE_CN(T, 16, false); }             \
  } while (0)
  if (bf16) BASE_CN_T(uint16_t);
  else BASE_CN_T(float);
#undef BASE_CN_T
#undef BASE_CN
  return hipGetLastError();
}

}  // namespace basek
