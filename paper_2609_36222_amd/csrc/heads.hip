// Norms of query and key heads with the rotation by position, and the same on the way
// into a paged cache:
//   t = g n(x)                      n(x) = x / sqrt(mean x^2 + eps)   (t = x without a gain)
//   (a, b) -> s (a cos w - b sin w, a sin w + b cos w)   for the pairs of t's first `rot`
// elements, w = position * inv_freq[pair]; the others pass.  All in fp32 and rounded
// once, but for the angle: a far position has no fp32 angle to speak of (at 10^6
// radians its step is 1/16), so the turns position * inv_freq / 2 pi are taken in fp64
// and their fraction goes on in fp32.
//
// Bound by memory: each head is read once and written once.  A lane holds 16 elements of
// a head, D / 16 lanes (rounded up to a power of two) a head, and a wavefront several
// heads of one row at a time, the next ones' loads in flight; the row's cosines and sines
// are computed once a wavefront, a pair a lane, and shared through LDS, while the first
// heads are on their way.  8191 rows of 16 + 16 fp32 heads of 128 (268 MB): 63.5 us, 4.2 TB/s
// of the 4.9 a large copy reaches; a cache filled by 205 MB of prompts 46.4 us, 4.4 TB/s; one
// row 3.2 us, of which the launch is most.
#include "common.hpp"
#include "internal.hpp"
#include "seq.hpp"

namespace basek {

namespace {

constexpr int HEAD_WAVES = 4;
constexpr int MAX_PAIRS = MAX_HEAD_D / 2;
// rows of a launch, a wavefront each: it has less than 2^32 work-items in all
constexpr long long LAUNCH_ROWS = 1LL << 25;

struct HeadsArgs {
  RopeArgs r;
  long long rows, row0, row1;   // the call's; the launch's: row0 .. row1 - 1
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

// What a lane has of a head.  MODE 1, rot and D multiples of 16: two runs of eight elements
// that are eight pairs' (a and b, or the pairs' one after another), all rotated or none.
// MODE 2, other heads with room for whole runs: the rotated elements and the others are cut
// apart, and the last lane of each takes runs that end with it; the first elements of such
// a run are another lane's too (both write the same values), and count once in the sum of
// squares.  MODE 0, the rest (less than 16 rotated elements, less than 8 others): eight pairs
// element by element.  (20000 rows of 40 heads with norms, 50 of 80 elements rotated, 256 MB:
// 84.8 us by runs, 209.8 element by element; 20 heads, 34 of 128: 74 against 192.)
struct Run {
  int p0, o1, o2;    // the first pair's number, the runs' places
  int dx, dy;        // how many of a run's first elements are another lane's
  bool inside, turned;
};
template <int MODE>
__device__ __forceinline__ Run run_of(int li, int D, int rot, bool interleaved) {
  Run r{};
  const int half = rot / 2;
  if constexpr (MODE != 2) {
    const bool halves = !interleaved && li * 8 < half;
    r.p0 = li * 8;
    r.o1 = halves ? r.p0 : 2 * r.p0;
    r.o2 = halves ? half + r.p0 : 2 * r.p0 + 8;
    r.inside = r.p0 < D / 2;
    r.turned = r.p0 < half;
  } else {
    const int turning = interleaved ? 0 : (half + 7) / 8, lane0 = li - turning;   // lanes with a and b apart
    if (lane0 < 0) {
      r.p0 = min(8 * li, half - 8);
      r.o1 = r.p0;
      r.o2 = half + r.p0;
      r.dx = r.dy = 8 * li - r.p0;
      r.inside = r.turned = true;
    } else {
      const int first = interleaved ? 0 : rot, n = D - first, at = first + 16 * lane0;
      r.inside = 16 * lane0 < n;
      r.o1 = n >= 16 ? min(at, D - 16) : first;
      r.o2 = n >= 16 ? r.o1 + 8 : D - 8;
      r.dx = n >= 16 ? min(at - r.o1, 8) : 0;
      r.dy = n >= 16 ? max(at - r.o1 - 8, 0) : 16 - n;
      r.p0 = r.o1 / 2;
      r.turned = interleaved && r.p0 < half;
    }
  }
  return r;
}
// lanes of a head
inline int run_lanes(int mode, int D, int rot, bool interleaved) {
  if (mode != 2 || interleaved) return (D + 15) / 16;
  return (rot / 2 + 7) / 8 + (D - rot + 15) / 16;
}
inline int run_mode(int D, int rot, bool interleaved) {
  if (D % 16 == 0 && rot % 16 == 0) return 1;
  if (interleaved) return D >= 16 ? 2 : 0;
  return rot >= 16 && (rot == D || D - rot >= 8) ? 2 : 0;
}

template <typename T, int MODE, bool CACHE>
__global__ __launch_bounds__(HEAD_WAVES * WAVE)
void k_heads(HeadsArgs a) {
  __shared__ float cs[HEAD_WAVES][2][MAX_PAIRS];
  const int w = wave_id_u(), lane = lane_id();
  const int job = blockIdx.x * HEAD_WAVES + w, at_row = job / a.split, part = job - at_row * a.split;
  const long long row = a.row0 + at_row;
  if (row >= a.row1) return;
  const int D = a.r.D, rot = a.r.rot, half = rot / 2;

  const int lph = a.lph, per = WAVE / lph, li = lane & (lph - 1), sub = lane / lph;
  const int pairs = D / 2;
  const Run run = run_of<MODE>(li, D, rot, a.r.interleaved);
  const int p0 = run.p0;
  const bool halves = !a.r.interleaved && run.turned;
  constexpr bool RUNS = MODE != 0;
  using Raw = decltype(raw8((const T *)nullptr));
  // a pass takes `per` heads; the first's runs are on their way while the angles are made,
  // the next one's while one is worked on
  auto source = [&](int pass) {
    const int h = pass * per + sub;
    const bool isq = h < a.Hq, isk = !isq && h < a.Hq + a.Hk;
    const HeadRows &in = isq ? a.q : isk ? a.k : a.v;
    return (const T *)in.p + row * in.row + (isq ? h : isk ? h - a.Hq : h - a.Hq - a.Hk) * in.head;
  };
  Raw r1{}, r2{};
  auto request = [&](int pass) {
    if (run.inside && pass * per + sub < a.heads) {
      const T *src = source(pass);
      r1 = raw8(src + run.o1);
      r2 = raw8(src + run.o2);
    }
  };
  if constexpr (RUNS) {
    if (part < a.passes) request(part);
  }

  int position = 0;
  long long kp = 0, vp = 0;      // the token's slot, head 0
  bool stored = false;           // the slot is there
  if constexpr (CACHE) {
    const int s = seq_of_row(a.b, (int)row);
    if (s < 0) return;           // behind the last sequence
    const SeqRows own = seq_rows(a.b.q_start[s], a.b.q_start[s + 1], a.b.kv_len[s], (int)a.rows,
                                 a.b.max_pages << a.c.shift);
    const long long at = (long long)own.kv - own.stop + row;   // (below 0: more new tokens than tokens)
    position = (int)at;
    if (at >= 0 && at < own.kv && row >= own.begin) {   // (at < kv: within the table's row)
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

  for (int pass = part; pass < a.passes; pass += a.split) {
    const int h = pass * per + sub;
    const bool have = run.inside && h < a.heads;
    const bool isq = h < a.Hq, isk = !isq && h < a.Hq + a.Hk;
    const int hl = isq ? h : isk ? h - a.Hq : h - a.Hq - a.Hk;
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
    float x[8], y[8];   // the runs at o1 and o2; in MODE 0 pair i is (x[i], y[i])
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.0f;
    if constexpr (RUNS) {
      if (have) {
        values8(r1, x);
        values8(r2, y);
      }
      if (pass + a.split < a.passes) request(pass + a.split);
    } else {
      if (have) {
        const T *src = source(pass);
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
        const float u = MODE == 2 && i < run.dx ? 0.0f : x[i], v = MODE == 2 && i < run.dy ? 0.0f : y[i];
        ss = __builtin_fmaf(u, u, ss);
        ss = __builtin_fmaf(v, v, ss);
      }
      if (lph > 16) ss = ss + xor_lane<16>(ss);
      if (lph > 8) ss = ss + xor_lane<8>(ss);
      if (lph > 4) ss = ss + xor_lane<4>(ss);
      if (lph > 2) ss = ss + xor_lane<2>(ss);
      if (lph > 1) ss = ss + xor_lane<1>(ss);
      if (gain && have) {
        const float m = ss / (float)D + a.r.eps;
        const float r = m > 0.0f ? 1.0f / __fsqrt_rn(m) : (m == 0.0f ? 0.0f : m);   // NaN stays NaN
        float gx[8], gy[8];
        if constexpr (RUNS) {
          values8(raw8(gain + run.o1), gx);
          values8(raw8(gain + run.o2), gy);
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
      if constexpr (RUNS) {
        if (run.turned) {
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
              if (MODE == 1 || p0 + i < half) {
                x[2 * i] = __builtin_fmaf(u, c[i], -(v * s[i]));
                x[2 * i + 1] = __builtin_fmaf(u, s[i], v * c[i]);
              }
              if (MODE == 1 || p0 + 4 + i < half) {
                y[2 * i] = __builtin_fmaf(e, c[4 + i], -(f * s[4 + i]));
                y[2 * i + 1] = __builtin_fmaf(e, s[4 + i], f * c[4 + i]);
              }
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
      if constexpr (RUNS) {
        store8(dst + run.o1, x);
        store8(dst + run.o2, y);
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
  a.r.interleaved = R.interleaved || R.rot == 0;
  const int mode = run_mode(R.D, R.rot, a.r.interleaved);
  a.lph = 1;
  while (a.lph < run_lanes(mode, R.D, R.rot, a.r.interleaved)) a.lph *= 2;
  a.passes = (a.heads * a.lph + WAVE - 1) / WAVE;
  const long long want = (16384 + rows - 1) / rows;   // (1 in calls of several launches)
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
#define BASE_HEADS(T, MODE)                                                                         \
  launch_k(cache ? k_heads<T, MODE, true> : k_heads<T, MODE, false>, grid, dim3(HEAD_WAVES *WAVE), 0, \
           st, a)
  for (a.row0 = 0; a.row0 < rows; a.row0 = a.row1) {
    a.row1 = a.row0 + LAUNCH_ROWS < rows ? a.row0 + LAUNCH_ROWS : rows;
    const dim3 grid((unsigned)(((a.row1 - a.row0) * a.split + HEAD_WAVES - 1) / HEAD_WAVES));
    if (bf16) { if (mode == 1) BASE_HEADS(uint16_t, 1); else if (mode == 2) BASE_HEADS(uint16_t, 2); else BASE_HEADS(uint16_t, 0); }
    else { if (mode == 1) BASE_HEADS(float, 1); else if (mode == 2) BASE_HEADS(float, 2); else BASE_HEADS(float, 0); }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
#undef BASE_HEADS
  return hipSuccess;
}

}  // namespace basek
