// RMS norms around a block, fused with its gate and the residual scale:
//   h' = a h + g * (w_post n(y))       (y itself without a post gain)
//   x' = w_pre n(h')                   n(v) = v / sqrt(mean v^2 + eps)
// over rows of d elements, everything in fp32 and each output rounded once (x'
// from h' before its rounding, so that the next block's input does not carry the
// residual stream's).  A row whose mean v^2 + eps is 0 has n(v) = 0.
//
// Bound by memory: y and h are read once, h' and x' written once, and the row
// lives in registers between the two means, EPT elements a thread.  A row of up to
// 128 elements is 16 lanes', of less than 256 32 lanes' and of up to 1024 one
// wavefront's (no barrier; 59,446 rows of 87 bf16 elements, a gate row each, 78 us with a
// wavefront a row, 13 so), a longer one a workgroup's, whose wavefronts join their
// sums through LDS; the threads follow from d (norm_threads).  A workgroup takes rows in turn, so that the
// gains, read once, stay in registers.  Accesses are 16 bytes at any element
// alignment: rows of odd length start anywhere, and global loads need no more
// than element alignment.  8191 rows of 5001 fp32 elements: 127 us, 5.2 TB/s, the rate of a
// large copy; with element accesses 226.  One row of 2048: 3.2 us, its two reductions and
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
    for (int e = 0; e < V; ++e) v[e] = 0.0f;
    if (left > 0) {   // (a branch an element would wait for each in turn)
      float q[V];
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = p[min(e, left - 1)];
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = e < left ? q[e] : 0.0f;
    }
  }
}
// 16 bytes of T as they lie, `left` elements of them in the row (zeros past it), and
// their values
__device__ __forceinline__ u32x4 norm_raw(const float *p, int left) {
  if (left >= 4) return __builtin_bit_cast(u32x4, reinterpret_cast<const Any16F *>(p)->v);
  u32x4 r = {0, 0, 0, 0};
  if (left > 0) {
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      const uint32_t q = __float_as_uint(p[min(e, left - 1)]);
      r[e] = e < left ? q : 0u;
    }
  }
  return r;
}
__device__ __forceinline__ u32x4 norm_raw(const uint16_t *p, int left) {
  if (left >= 8) return reinterpret_cast<const Any16H *>(p)->v;
  u32x4 r = {0, 0, 0, 0};
  if (left > 0) {
#pragma unroll
    for (int e = 0; e < 7; ++e) {
      const uint32_t q = p[min(e, left - 1)];
      r[e / 2] |= (e < left ? q : 0u) << (16 * (e & 1));
    }
  }
  return r;
}
__device__ __forceinline__ void norm_values(u32x4 r, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void norm_values(u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
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
      q[i] = (uint32_t)f32_to_bf16_any(v[2 * i]) | ((uint32_t)f32_to_bf16_any(v[2 * i + 1]) << 16);
    reinterpret_cast<Any16H *>(p)->v = q;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < left) p[e] = f32_to_bf16_any(v[e]);
  }
}

// Elements a thread and threads a row: the same for k_norm and k_combine_norm, so
// that their sums have one order and the block call the bits of its parts.  (From 513
// to 1024 a row is one wavefront's with 16; with 8 and two wavefronts, us: 255 rows 4.7
// -> 3.9; bf16, 8191 rows of 640 13.9 -> 11.4, of 1024 14.4 -> 14.3, 40,000 of 640 52.6 ->
// 43.9; fp32, 8191 of 640 16.4 -> 14.7, 40,000 of 640 81.1 -> 81.0, of 1000 126 -> 131.)
__host__ __device__ inline int norm_ept(int d) { return d <= 512 || (d > 1024 && d <= 2048) ? 8 : 16; }
__host__ __device__ inline int norm_threads(int d) {
  const int per = WAVE * norm_ept(d);
  return (d + per - 1) / per * WAVE;
}
static_assert(MAX_NORM_D <= 16 * 1024, "a row in one workgroup's registers");

// Sum over the row's LPR lanes or (0) its workgroup, the same value in all of them: a
// butterfly in the wavefront, then the wavefronts' sums in ascending order.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float *red) {
  if constexpr (LPR == 0 || LPR > 32) v = v + xor_lane<32>(v);
  if constexpr (LPR == 0 || LPR > 16) v = v + xor_lane<16>(v);
  v = v + xor_lane<8>(v);
  v = v + xor_lane<4>(v);
  v = v + xor_lane<2>(v);
  v = v + xor_lane<1>(v);
  if constexpr (LPR == 0) {
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
// WIN, for rows that V does not divide: the last piece starts V elements before the
// row's end, and the elements it has in common with the piece before it are left out
// of the sums and stored twice, with the same values.  (By elements, one lane's loads
// and stores hold up its workgroup: 8191 rows of 5004 bf16 elements 127 us, now 66.)
template <typename T, int EPT, int LPR, bool WIN>
struct NormRow {
  static constexpr int V = 16 / sizeof(T), Q = EPT / V;
  float post[EPT], pre[EPT], gate[EPT];
  int tid, threads, d, first[Q], twice[Q];
  __device__ NormRow(int tid_, int threads_, int d_) : tid(tid_), threads(threads_), d(d_) {
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const int c = (i * threads + tid) * V;
      first[i] = WIN && d >= V && c < d ? min(c, d - V) : c;
      twice[i] = c - first[i];
    }
  }
  template <typename P>
  __device__ void load(const P *p, float (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) norm_load<V>(p + first[i], d - first[i], &v[i * V]);
  }
  // a row of T and its values
  __device__ void fetch(const T *p, u32x4 (&r)[Q]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) r[i] = norm_raw(p + first[i], d - first[i]);
  }
  __device__ void values(const u32x4 (&r)[Q], float (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) norm_values(r[i], *reinterpret_cast<float (*)[V]>(&v[i * V]));
  }
  __device__ void store(T *p, const float (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) norm_store<V>(p + first[i], d - first[i], &v[i * V]);
  }
  __device__ float rstd(const float (&v)[EPT], float eps, float *red) const {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const float q = WIN && i % V < twice[i / V] ? 0.0f : v[i];
      ss = __builtin_fmaf(q, q, ss);
    }
    return row_rstd(row_sum<LPR>(ss, red), d, eps);
  }
  // the parameters that every row shares
  __device__ void params(const NormArgs &a, bool pre_needed) {
    if (a.post) load(a.post, post);
    if (a.gate && a.gate_ld == 0) load(a.gate, gate);
    if (pre_needed) load(a.pre, pre);
  }
  // one row (have: there is one) from h (v) and, with HAS_Y, the block's output (s)
  template <bool HAS_Y>
  __device__ void run(const NormArgs &a, float (&v)[EPT], float (&s)[EPT], T *ho, T *xo, float *red,
                      bool have = true) {
    if (HAS_Y) {
      const float r = a.post ? rstd(s, a.eps, red) : 1.0f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        float t = s[i];
        if (a.post) t = t * r * post[i];
        if (a.gate) t = t * gate[i];
        v[i] = __builtin_fmaf(a.scale, v[i], t);
      }
      if (ho && have) store(ho, v);
    }
    if (xo) {
      const float r = rstd(v, a.eps, red + 16);
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] = v[i] * r * pre[i];
      if (have) store(xo, v);
    }
  }
};

// ho may be h or y and xo may be y or h: a row's elements are read before any of it is
// written.
template <typename T, int EPT, int LPR, bool WIN, bool HAS_Y>
__global__ __launch_bounds__(LPR > 0 ? 256 : 1024)
void k_norm(NormArgs a, long long rows, const T *y, long long y_ld, const T *h, long long h_ld,
            T *ho, long long ho_ld, T *xo, long long xo_ld) {
  __shared__ float red[LPR > 0 ? 1 : 32];
  using Row = NormRow<T, EPT, LPR, WIN>;
  constexpr int PER = LPR > 0 ? WAVE / LPR : 1;   // rows a wavefront or workgroup
  Row n(LPR > 0 ? lane_id() % (LPR > 0 ? LPR : 1) : (int)threadIdx.x,
        LPR > 0 ? LPR : (int)blockDim.x, a.d);
  const int sub = LPR > 0 ? lane_id() / (LPR > 0 ? LPR : 1) : 0;
  const int waves = LPR > 0 ? (int)blockDim.x / WAVE : 1;
  const long long step = (long long)gridDim.x * waves * PER;
  long long row0 = ((long long)blockIdx.x * waves + (LPR > 0 ? wave_id_u() : 0)) * PER;
  n.params(a, xo != nullptr);
  for (; row0 < rows; row0 += step) {
    const bool have = row0 + sub < rows;
    const long long row = have ? row0 + sub : rows - 1;
    float v[EPT], s[EPT];
    u32x4 hr[Row::Q], yr[Row::Q];
    n.fetch(h + row * h_ld, hr);
    if (HAS_Y) {
      n.fetch(y + row * y_ld, yr);
      if (a.gate && a.gate_ld != 0) n.load(a.gate + row * a.gate_ld, n.gate);
    }
    // in place: a piece is read before another wavefront writes its neighbour
    if (LPR == 0 && WIN) __syncthreads();
    n.values(hr, v);
    if (HAS_Y) n.values(yr, s);
    n.template run<HAS_Y>(a, v, s, ho ? ho + row * ho_ld : nullptr, xo ? xo + row * xo_ld : nullptr,
                          red, have);
    if (LPR == 0) __syncthreads();   // red is free for the next row
  }
}

// The layer's combine and the norm behind it: y_t = sum_j pairbuf[pair_of[t][j]]
// in j order, rounded to T as base_decode_layer writes it, then the row.
// SPLIT: a pair's row is the sum of `shares` rows `stride` apart, in their order.
template <typename T, int EPT, int LPR, bool SPLIT>
__global__ __launch_bounds__(LPR > 0 ? LPR : 1024)
void k_combine_norm(NormArgs a, int kc, const int32_t *__restrict__ pair_of,
                    const float *__restrict__ pairbuf, int shares, size_t stride, const T *h, T *ho,
                    T *xo) {
  __shared__ float red[LPR > 0 ? 1 : 32];
  constexpr int GROUP = 4;   // ranks whose rows are in flight together
  NormRow<T, EPT, LPR, false> n(threadIdx.x, blockDim.x, a.d);
  const size_t t = blockIdx.x;
  const int d = a.d;
  float v[EPT], s[EPT];
  u32x4 hr[EPT * sizeof(T) / 16];
  n.fetch(h + t * d, hr);
  n.values(hr, v);
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
    for (int g = 0; g < GROUP; ++g) n.load(pairbuf + (size_t)max(p[g], 0) * d, o[g]);
#pragma unroll
    for (int g = 0; g < GROUP; ++g) {
      if (p[g] < 0) continue;   // a routed rank the token does not execute
      for (int q = 1; SPLIT && q < shares; ++q) {
        float e[EPT];
        n.load(pairbuf + q * stride + (size_t)p[g] * d, e);
#pragma unroll
        for (int i = 0; i < EPT; ++i) o[g][i] = o[g][i] + e[i];
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[i] = s[i] + o[g][i];
    }
  }
  if (a.gate && a.gate_ld != 0) n.load(a.gate + t * a.gate_ld, n.gate);
  n.params(a, xo != nullptr);
#pragma unroll
  for (int i = 0; i < EPT; ++i) s[i] = sizeof(T) == 2 ? bf16_to_f32(f32_to_bf16(s[i])) : s[i];
  n.template run<true>(a, v, s, ho ? ho + t * d : nullptr, xo ? xo + t * d : nullptr, red);
}

hipError_t launch_norm(bool bf16, int d, float eps, float scale, const float *post, const float *gate,
                       long long gate_ld, const float *pre, long long rows, const void *y,
                       long long y_ld, const void *h, long long h_ld, void *ho, long long ho_ld,
                       void *xo, long long xo_ld, int n_cu, hipStream_t st) {
  // (a norm without y reads no parameter of the block's, pointers among them)
  const NormArgs a{d, eps, scale, y ? post : nullptr, y ? gate : nullptr, pre, gate_ld};
  const int V = bf16 ? 8 : 4, lpr = d <= 128 ? 16 : d < 256 ? 32 : d <= 16 * WAVE ? WAVE : 0;
  // rows that V does not divide, in workgroups of more threads: with 16 elements a
  // thread the registers spill (past 8192 elements there are not as many threads)
  const bool win = d % V != 0 && d <= 8192;
  const int ept = win && lpr == 0 ? 8 : norm_ept(d);
  const int threads = lpr ? 4 * WAVE : (d + WAVE * ept - 1) / (WAVE * ept) * WAVE;
  const int per = lpr ? 4 * (WAVE / lpr) : 1;
  // as many wavefronts a CU as the registers allow, in workgroups that stride over the
  // rows (8191 rows of 5001 bf16 elements with 16 instead of 24: 121 us against 77)
  const int cu_waves = ept == 8 && lpr == 0 ? 24 : 16;
  const long long most = (long long)n_cu * (cu_waves * WAVE / threads > 0 ? cu_waves * WAVE / threads : 1);
  const long long blocks = (rows + per - 1) / per;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
#define BASE_NORM(T, EPT, LPR, WIN)                                                               \
  launch_k(y ? k_norm<T, EPT, LPR, WIN, true> : k_norm<T, EPT, LPR, WIN, false>, grid,            \
           dim3(threads), 0, st, a, rows, (const T *)y, y_ld, (const T *)h, h_ld, (T *)ho, ho_ld, \
           (T *)xo, xo_ld)
#define BASE_NORM_W(T, EPT, LPR)                                                                 \
  do { if (win) BASE_NORM(T, EPT, LPR, true); else BASE_NORM(T, EPT, LPR, false); } while (0)
#define BASE_NORM_T(T)                                                                           \
  do {                                                                                           \
    if (lpr == 16) BASE_NORM(T, 8, 16, true);                                                    \
    else if (lpr == 32) BASE_NORM(T, 8, 32, true);                                               \
    else if (lpr) { if (ept == 8) BASE_NORM_W(T, 8, WAVE); else BASE_NORM_W(T, 16, WAVE); }      \
    else if (ept == 8) BASE_NORM_W(T, 8, 0);                                                     \
    else BASE_NORM(T, 16, 0, false);                                                             \
  } while (0)
  if (bf16) BASE_NORM_T(uint16_t);
  else BASE_NORM_T(float);
#undef BASE_NORM_T
#undef BASE_NORM_W
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
#define BASE_CN(T, EPT, LPR)                                                                     \
  launch_k(shares > 1 ? k_combine_norm<T, EPT, LPR, sizeof(T) == 2>                              \
                      : k_combine_norm<T, EPT, LPR, false>,                                      \
           dim3(B), dim3(threads), 0, st, a, kc, pair_of, pairbuf, shares, stride, (const T *)h, \
           (T *)ho, (T *)xo)
#define BASE_CN_T(T)                                                                             \
  do {                                                                                           \
    if (threads > WAVE) { if (norm_ept(d) == 8) BASE_CN(T, 8, 0); else BASE_CN(T, 16, 0); }      \
    else { if (norm_ept(d) == 8) BASE_CN(T, 8, WAVE); else BASE_CN(T, 16, WAVE); }               \
  } while (0)
  if (bf16) BASE_CN_T(uint16_t);
  else BASE_CN_T(float);
#undef BASE_CN_T
#undef BASE_CN
  return hipGetLastError();
}

}  // namespace basek
