// Norms of query and key heads with the rotation by position, and the same on the way
// into a paged cache:
//   t = g n(x)                      n(x) = x / sqrt(mean x^2 + eps)   (t = x without a gain)
//   (a, b) -> s (a cos w - b sin w, a sin w + b cos w)   for the pairs of t's first `rot`
// elements, w = position * inv_freq[pair]; the others pass.  All in fp32 and rounded
// once, but for the angle: a far position has no fp32 angle to speak of (at 10^6
// radians its step is 1/16), so the turns position * inv_freq / 2 pi are taken in fp64
// and their fraction goes on in fp32.
//
// Bound by memory: each head is read once and written once.  A lane holds eight pairs of
// a head, D / 16 lanes (rounded up to a power of two) a head, and a wavefront several
// heads of one row at a time, the next ones' loads in flight; the row's cosines and sines
// are computed once a wavefront, a pair a lane, and shared through LDS.
#include "common.hpp"
#include "internal.hpp"
#include "seq.hpp"

namespace basek {

namespace {

constexpr int HEAD_WAVES = 4;
constexpr int MAX_PAIRS = MAX_HEAD_D / 2;

struct HeadsArgs {
  RopeArgs r;
  long long rows;
  const int32_t *pos;
  int Hq, Hk, heads, lph, passes, split;   // heads: with the values; split: wavefronts a row
  HeadRows q, qo, k, ko, v;
  KvCache c;
  KvBatch b;
};

// cos and sin of 2 pi t for a fraction of a turn |t| <= 1/2: the eighth around the
// nearest quarter by the Taylor series (error below 2^-27 at pi / 4)
__device__ __forceinline__ void turn(float t, float &c, float &s) {
  const float n = __builtin_rintf(4.0f * t);
  const float x = (t - 0.25f * n) * 6.2831853071795865f;   // exact difference
  const float z = x * x;
  float sp = 1.0f / 362880.0f;
  sp = __builtin_fmaf(sp, z, -1.0f / 5040.0f);
  sp = __builtin_fmaf(sp, z, 1.0f / 120.0f);
  sp = __builtin_fmaf(sp, z, -1.0f / 6.0f);
  const float sx = __builtin_fmaf(x * z, sp, x);
  float cp = -1.0f / 3628800.0f;
  cp = __builtin_fmaf(cp, z, 1.0f / 40320.0f);
  cp = __builtin_fmaf(cp, z, -1.0f / 720.0f);
  cp = __builtin_fmaf(cp, z, 1.0f / 24.0f);
  cp = __builtin_fmaf(cp, z, -0.5f);
  const float cx = __builtin_fmaf(z, cp, 1.0f);
  const int q = (int)n & 3;
  const float a = (q & 1) ? sx : cx, b = (q & 1) ? cx : sx;
  c = (q == 1 || q == 2) ? -a : a;
  s = (q >= 2) ? -b : b;
}

struct __attribute__((packed, aligned(4))) Any16F { f32x4 v; };
struct __attribute__((packed, aligned(2))) Any16H { u32x4 v; };

// eight consecutive elements as they lie, at any element alignment
struct Raw8F { f32x4 lo, hi; };
__device__ __forceinline__ Raw8F raw8(const float *p) {
  return {reinterpret_cast<const Any16F *>(p)->v, reinterpret_cast<const Any16F *>(p + 4)->v};
}
__device__ __forceinline__ u32x4 raw8(const uint16_t *p) { return reinterpret_cast<const Any16H *>(p)->v; }
__device__ __forceinline__ void values8(const Raw8F &r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = r.lo[i]; v[4 + i] = r.hi[i]; }
}
__device__ __forceinline__ void values8(const u32x4 &r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  reinterpret_cast<Any16F *>(p)->v = f32x4{v[0], v[1], v[2], v[3]};
  reinterpret_cast<Any16F *>(p + 4)->v = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
  u32x4 q;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    q[i] = (uint32_t)f32_to_bf16_any(v[2 * i]) | ((uint32_t)f32_to_bf16_any(v[2 * i + 1]) << 16);
  reinterpret_cast<Any16H *>(p)->v = q;
}
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = f32_to_bf16_any(v); }

// VEC: rot and D are multiples of 16, so that a lane's eight pairs are two runs of eight
// elements, all rotated or none.
template <typename T, bool VEC, bool CACHE>
__global__ __launch_bounds__(HEAD_WAVES * WAVE)
void k_heads(HeadsArgs a) {
  __shared__ float cs[HEAD_WAVES][2][MAX_PAIRS];
  const int w = wave_id_u(), lane = lane_id();
  const long long job = (long long)blockIdx.x * HEAD_WAVES + w;
  const long long row = job / a.split;
  const int part = (int)(job - row * a.split);
  if (row >= a.rows) return;
  const int D = a.r.D, rot = a.r.rot, half = rot / 2;

  int position = 0;
  long long kp = 0, vp = 0;      // the token's slot, head 0
  bool stored = false;           // the slot is there
  if constexpr (CACHE) {
    const int s = seq_of_row(a.b, (int)row);
    if (s < 0) return;           // behind the last sequence
    const int start = a.b.q_start[s], stop = a.b.q_start[s + 1], kv = a.b.kv_len[s];
    const long long at = (long long)kv - stop + row;   // row - start new tokens before it
    position = (int)at;
    if (at >= 0 && at < kv && row >= start && (at >> a.c.shift) < a.b.max_pages) {
      const int page = a.b.table[s * a.b.table_ld + (at >> a.c.shift)];
      if ((unsigned)page < (unsigned)a.c.n_pages) {
        const long long slot = at & ((1LL << a.c.shift) - 1);
        kp = page * a.c.k_page + slot * a.c.k_slot;
        vp = page * a.c.v_page + slot * a.c.v_slot;
        stored = true;
      }
    }
  }
  if (a.pos) position = a.pos[row];
  for (int i = lane; i < half; i += WAVE) {
    const double t = (double)position * (double)a.r.inv[i] * 0.15915494309189533577;   // 1 / 2 pi
    float c, s;
    turn((float)(t - __builtin_rint(t)), c, s);
    cs[w][0][i] = c * a.r.scale;
    cs[w][1][i] = s * a.r.scale;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

  const int lph = a.lph, per = WAVE / lph, li = lane & (lph - 1), sub = lane / lph;
  const int pairs = D / 2, p0 = li * 8;
  const bool inside = p0 < pairs;            // the lane holds pairs of the head
  const bool halves = !a.r.interleaved && p0 < half;
  const int o1 = halves ? p0 : 2 * p0, o2 = halves ? half + p0 : 2 * p0 + 8;   // VEC

  for (int pass = part; pass < a.passes; pass += a.split) {
    const int h = pass * per + sub;
    const bool have = inside && h < a.heads;
    const bool isq = h < a.Hq, isk = !isq && h < a.Hq + a.Hk;
    const int hl = isq ? h : isk ? h - a.Hq : h - a.Hq - a.Hk;
    const HeadRows &in = isq ? a.q : isk ? a.k : a.v;
    const T *src = (const T *)in.p + row * in.row + hl * in.head;
    T *dst;
    bool write = have;
    if (!CACHE || isq) {
      const HeadRows &out = isq ? a.qo : a.ko;
      dst = (T *)out.p + row * out.row + hl * out.head;
    } else {
      dst = isk ? (T *)a.c.k + kp + hl * a.c.k_head : (T *)a.c.v + vp + hl * a.c.v_head;
      write = have && stored;
    }
    const float *gain = isq ? a.r.q_gain : isk ? a.r.k_gain : nullptr;
    float x[8], y[8];   // VEC: the runs at o1 and o2; else pair i is (x[i], y[i])
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.0f;
    if constexpr (VEC) {
      if (have) {
        const auto r1 = raw8(src + o1), r2 = raw8(src + o2);
        values8(r1, x);
        values8(r2, y);
      }
    } else {
      if (have) {
        T u[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int p = min(p0 + i, pairs - 1);
          const bool split = !a.r.interleaved && p < half;
          u[i] = src[split ? p : 2 * p];
          u[8 + i] = src[split ? half + p : 2 * p + 1];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = p0 + i < pairs ? value(u[i]) : 0.0f;
          y[i] = p0 + i < pairs ? value(u[8 + i]) : 0.0f;
        }
      }
    }
    if (a.r.q_gain || a.r.k_gain) {
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = __builtin_fmaf(x[i], x[i], ss);
        ss = __builtin_fmaf(y[i], y[i], ss);
      }
      if (lph > 8) ss = ss + xor_lane<8>(ss);
      if (lph > 4) ss = ss + xor_lane<4>(ss);
      if (lph > 2) ss = ss + xor_lane<2>(ss);
      if (lph > 1) ss = ss + xor_lane<1>(ss);
      if (gain && have) {
        const float m = ss / (float)D + a.r.eps;
        const float r = m > 0.0f ? 1.0f / __fsqrt_rn(m) : (m == 0.0f ? 0.0f : m);   // NaN stays NaN
        float gx[8], gy[8];
        if constexpr (VEC) {
          values8(raw8(gain + o1), gx);
          values8(raw8(gain + o2), gy);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int p = min(p0 + i, pairs - 1);
            const bool split = !a.r.interleaved && p < half;
            gx[i] = gain[split ? p : 2 * p];
            gy[i] = gain[split ? half + p : 2 * p + 1];
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = x[i] * r * gx[i];
          y[i] = y[i] * r * gy[i];
        }
      }
    }
    if (isq || isk) {
      if constexpr (VEC) {
        if (p0 < half) {
          const float *c = &cs[w][0][p0], *s = &cs[w][1][p0];
          if (halves) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float u = x[i], v = y[i];
              x[i] = __builtin_fmaf(u, c[i], -(v * s[i]));
              y[i] = __builtin_fmaf(u, s[i], v * c[i]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float u = x[2 * i], v = x[2 * i + 1], e = y[2 * i], f = y[2 * i + 1];
              x[2 * i] = __builtin_fmaf(u, c[i], -(v * s[i]));
              x[2 * i + 1] = __builtin_fmaf(u, s[i], v * c[i]);
              y[2 * i] = __builtin_fmaf(e, c[4 + i], -(f * s[4 + i]));
              y[2 * i + 1] = __builtin_fmaf(e, s[4 + i], f * c[4 + i]);
            }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (p0 + i < half) {
            const float c = cs[w][0][p0 + i], s = cs[w][1][p0 + i], u = x[i], v = y[i];
            x[i] = __builtin_fmaf(u, c, -(v * s));
            y[i] = __builtin_fmaf(u, s, v * c);
          }
        }
      }
    }
    if (write) {
      if constexpr (VEC) {
        store8(dst + o1, x);
        store8(dst + o2, y);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int p = p0 + i;
          if (p >= pairs) continue;
          const bool split = !a.r.interleaved && p < half;
          put(dst + (split ? p : 2 * p), x[i]);
          put(dst + (split ? half + p : 2 * p + 1), y[i]);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_heads(bool bf16, const RopeArgs &R, long long rows, const int32_t *pos, int Hq,
                        HeadRows q, HeadRows q_out, int Hk, HeadRows k, HeadRows k_out,
                        HeadRows v, const KvCache *cache, const KvBatch *batch, hipStream_t st) {
  HeadsArgs a{};
  a.r = R;
  a.rows = rows;
  a.pos = pos;
  a.Hq = Hq;
  a.Hk = Hk;
  a.heads = Hq + Hk + (cache ? Hk : 0);
  a.lph = 1;
  while (a.lph * 16 < R.D) a.lph *= 2;
  a.passes = (a.heads * a.lph + WAVE - 1) / WAVE;
  const long long want = (16384 + rows - 1) / rows;
  a.split = (int)(want < a.passes ? want : a.passes);
  a.q = q;
  a.qo = q_out;
  a.k = k;
  a.ko = k_out;
  a.v = v;
  if (cache) {
    a.c = *cache;
    a.b = *batch;
  }
  const dim3 grid((unsigned)((rows * a.split + HEAD_WAVES - 1) / HEAD_WAVES));
  const bool vec = R.D % 16 == 0 && R.rot % 16 == 0;
#define BASE_HEADS(T, V)                                                                        \
  launch_k(cache ? k_heads<T, V, true> : k_heads<T, V, false>, grid, dim3(HEAD_WAVES *WAVE), 0, \
           st, a)
  if (bf16) { if (vec) BASE_HEADS(uint16_t, true); else BASE_HEADS(uint16_t, false); }
  else { if (vec) BASE_HEADS(float, true); else BASE_HEADS(float, false); }
#undef BASE_HEADS
  return hipGetLastError();
}

}  // namespace basek
