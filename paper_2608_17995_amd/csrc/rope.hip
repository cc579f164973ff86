// RMS norm of each head's query and key and the rotation by their positions,
// in one pass over the rows, and its backward pass.
//
// Forward, for a head's d values x:  n = x rstd, rstd = (avg x^2 + eps)^-1/2,
// y = n g, and each pair (a, b) of y's first `rot` elements becomes
// (a cos t - b sin t, a sin t + b cos t), t = pos[axis] pos_scale freq[pair].
// Backward, from e = the gradient turned back by -t:
//   dg = sum over rows and heads of e n,  dx = rstd (e g - n avg(e g n)).
// A lane holds four pairs of a head: 16 (8) lanes make a head of 128 (64), a
// wave four (eight) heads of one row.  The lane's four sines and cosines are
// made once and used for all heads of the row.
// Angles are taken in 64 bits and reduced to a fraction of a turn, so that far
// positions lose nothing.
#include <math.h>

#include "kernels.h"

namespace avits {
namespace {

constexpr int kMaxAxes = 4;

struct RopeArgs {
  const void* x[2];    // queries and keys (backward: before the norm)
  const void* dy[2];   // backward: gradients of the rotated rows
  void* out[2];        // rotated rows (backward: gradients of x)
  int64_t x_ld[2], dy_ld[2], out_ld[2];
  const void* g[2];
  float* part;         // backward: [workgroup][2][d] sums of the gains' gradients
  const int32_t* pos;
  const double* freq;
  double pos_scale;
  int64_t M;
  int H[2];            // heads of the queries and of the keys
  int rot, axes;
  int end[kMaxAxes];   // pairs before the end of each axis
  float eps;           // 0: no norm
  int64_t per;         // rows of one wave
  int parts;           // waves that share a row's heads
};

// Sine and cosine of f turns, |f| <= 1/2: fp32 rows take the library's, bf16
// rows the instruction's, whose error (below 2^-20) is far below their own step.
template <typename T>
__device__ __forceinline__ void turn_of(float f, float& s, float& c) {
  if constexpr (sizeof(T) == 4) {
    sincospif(2.f * f, &s, &c);
  } else {
    s = __builtin_amdgcn_sinf(f);
    c = __builtin_amdgcn_cosf(f);
  }
}

// Where a lane's eight elements lie in their head.
// HALVES: pair p is (p, p + rot / 2), else (2 p, 2 p + 1); the elements past
// rot, which are not turned, pair up as (0, 4), (1, 5), ... of each eight with
// whole vectors, as neighbours otherwise.
template <typename T, bool HALVES, bool VEC>
struct Lane {
  uint32_t a[VEC ? 1 : 4], b[VEC ? 1 : 4];
  // head: where the lane's head of a step starts.
  __device__ __forceinline__ Lane(int p0, int rot, int head) {
    if constexpr (VEC) {
      a[0] = 2 * p0;
      b[0] = 2 * p0 + 4;
      if (HALVES && p0 < rot / 2) {
        a[0] = p0;
        b[0] = p0 + rot / 2;
      }
      a[0] += head;
      b[0] += head;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i;
        const bool split = HALVES && p < rot / 2;
        a[i] = head + (split ? p : 2 * p);
        b[i] = head + (split ? p + rot / 2 : 2 * p + 1);
      }
    }
  }
  // Eight elements as they lie in memory.
  static constexpr int kWords = VEC ? 2 * sizeof(T) : 8;
  struct Raw {
    uint32_t w[kWords];
  };
  __device__ __forceinline__ Raw fetch(const T* p) const {
    Raw r;
    if constexpr (!VEC) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) r.w[i] = __float_as_uint(p[a[i]]), r.w[4 + i] = __float_as_uint(p[b[i]]);
        else r.w[i] = uint32_t(p[a[i]]) << 16, r.w[4 + i] = uint32_t(p[b[i]]) << 16;
      }
    } else if constexpr (sizeof(T) == 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + a[0]), y = *reinterpret_cast<const u32x4*>(p + b[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[i] = x[i], r.w[4 + i] = y[i];
    } else if constexpr (HALVES) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(p + a[0]), y = *reinterpret_cast<const u32x2*>(p + b[0]);
      r.w[0] = x[0], r.w[1] = x[1], r.w[2] = y[0], r.w[3] = y[1];
    } else {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + a[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[i] = x[i];
    }
    return r;
  }
  // The first and the second elements of the four pairs.
  __device__ __forceinline__ static void unpack(const Raw& r, float* va, float* vb) {
    float v[8];
    if constexpr (kWords == 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      va[i] = v[HALVES || !VEC ? i : 2 * i];
      vb[i] = v[HALVES || !VEC ? 4 + i : 2 * i + 1];
    }
  }
  __device__ __forceinline__ static void put4(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    else *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
  }
  __device__ __forceinline__ void store(T* p, const float* va, const float* vb) const {
    if constexpr (VEC) {
      if constexpr (HALVES) {
        put4(p + a[0], va);
        put4(p + b[0], vb);
      } else if constexpr (sizeof(T) == 4) {
        const float v[8] = {va[0], vb[0], va[1], vb[1], va[2], vb[2], va[3], vb[3]};
        put4(p + a[0], v);
        put4(p + a[0] + 4, v + 4);
      } else {
        *reinterpret_cast<u32x4*>(p + a[0]) =
            u32x4{pack_bf2(va[0], vb[0]), pack_bf2(va[1], vb[1]), pack_bf2(va[2], vb[2]), pack_bf2(va[3], vb[3])};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st(p, a[i], va[i]);
        st(p, b[i], vb[i]);
      }
    }
  }
};

// The turns of a row's four pairs of this lane; `on` of them turn, the first ones.
template <typename T>
struct Turns {
  double f[4];  // turns to a position
  int axis[4], on;
  __device__ __forceinline__ Turns(const RopeArgs& a, int p0) {
    on = std::min(4, std::max(0, a.rot / 2 - p0));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = 0.0;
      axis[i] = 0;
      if (i < on) {
        f[i] = a.freq[p0 + i] * a.pos_scale * 0.15915494309189533577;
#pragma unroll
        for (int x = 0; x < kMaxAxes - 1; ++x) axis[i] += x < a.axes - 1 && p0 + i >= a.end[x] ? 1 : 0;
      }
    }
  }
  __device__ __forceinline__ void at(const RopeArgs& a, int64_t row, float* s, float* c) const {
    if (on == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double turns = double(a.pos[row * a.axes + axis[i]]) * f[i];
      turn_of<T>(float(turns - rint(turns)), s[i], c[i]);
    }
  }
  // (a, b) to (a c - b s, a s + b c).  Elements that do not turn are no pair: what one holds is not the other's.
  __device__ __forceinline__ void turn(float* va, float* vb, const float* s, const float* c) const {
    if (on == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = va[i] * c[i] - vb[i] * s[i], y = va[i] * s[i] + vb[i] * c[i];
      if (on == 4 || i < on) {
        va[i] = x;
        vb[i] = y;
      }
    }
  }
};

// The part of the queries' (or keys') steps, kHPW heads each, that falls to part p of n.
struct Span {
  int lo, up;
  __device__ __forceinline__ Span(int heads, int hpw, int p, int n) {
    const int steps = (heads + hpw - 1) / hpw;
    lo = steps * p / n;
    up = steps * (p + 1) / n;
  }
};

template <typename T, int DH, bool HALVES, bool VEC>
__device__ __forceinline__ void load_gain(const Lane<T, HALVES, VEC>& at, uint32_t head, const void* gain, float* ga, float* gb) {
  const T* p = static_cast<const T*>(gain);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ga[i] = gb[i] = 1.f;
    if (p) {  // the gain itself need not lie on 16 bytes
      ga[i] = ld(p, (VEC ? (HALVES ? at.a[0] + i : at.a[0] + 2 * i) : at.a[VEC ? 0 : i]) - head);
      gb[i] = ld(p, (VEC ? (HALVES ? at.b[0] + i : at.a[0] + 2 * i + 1) : at.b[VEC ? 0 : i]) - head);
    }
  }
}

// Bound by HBM: each row is read and written once.  The first kU steps of the queries and of the keys are under
// way together (16 heads of 128 each: the whole row), as they lie in memory, to hold few registers.  16896 rows of 16 + 16
// heads of 128 in bf16, 277 MB: 50 us, 5.5 TB/s (a call 58; with one step
// after another 73); one row 4.3 us, a launch.
template <typename T, int DH, bool HALVES, bool VEC>
__global__ __launch_bounds__(256) void qk_rotate_kernel(const RopeArgs a) {
  constexpr int kLPH = DH / 8, kHPW = kWave / kLPH, kU = 4;  // lanes to a head, heads to a step, steps at once
  typedef Lane<T, HALVES, VEC> At;
  const int lane = threadIdx.x % kWave, p0 = 4 * (lane % kLPH), sub = lane / kLPH;
  const int64_t wave = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int part = int(wave % a.parts);
  const int64_t first = wave / a.parts * a.per, last = std::min(a.M, first + a.per);
  if (first >= last) return;
  const At at(p0, a.rot, sub * DH);
  const Turns<T> turns(a, p0);
  const Span span[2] = {Span(a.H[0], kHPW, part, a.parts), Span(a.H[1], kHPW, part, a.parts)};
  for (int64_t row = first; row < last; ++row) {
    typename At::Raw raw[2][kU];
    auto fetch = [&](int w, int st) {
      const T* in = static_cast<const T*>(a.x[w]) + row * a.x_ld[w];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u < span[w].up && t < a.H[w]) raw[w][u] = at.fetch(in + (st + u) * (kHPW * DH));
      }
    };
#pragma unroll
    for (int w = 0; w < 2; ++w) fetch(w, span[w].lo);
    float s[4], c[4];
    turns.at(a, row, s, c);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (span[w].lo >= span[w].up) continue;
      float ga[4], gb[4];
      load_gain<T, DH>(at, sub * DH, a.g[w], ga, gb);
      T* out = static_cast<T*>(a.out[w]) + row * a.out_ld[w];
      for (int st = span[w].lo; st < span[w].up; st += kU) {
        if (st > span[w].lo) fetch(w, st);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int t = (st + u) * kHPW + sub;
          if (st + u >= span[w].up || t >= a.H[w]) continue;
          float va[4], vb[4];
          at.unpack(raw[w][u], va, vb);
          if (a.eps > 0.f) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += va[i] * va[i] + vb[i] * vb[i];
            const float r = rsqrtf(group_sum(sum, kLPH) * (1.f / DH) + a.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              va[i] *= r * ga[i];
              vb[i] *= r * gb[i];
            }
          }
          turns.turn(va, vb, s, c);
          at.store(out + (st + u) * (kHPW * DH), va, vb);
        }
      }
    }
  }
}

// The backward pass reads x and the gradient and writes dx.  A wave has consecutive rows, whose shares of the gains' gradients
// it keeps in registers; as many waves as the chip holds, so that there are few sums for the second launch.  4608 rows of
// 16 + 16 heads of 128 in bf16, 113 MB: 25 to 27 us, 4.2 to 4.5 TB/s, and 3.9 for the sums (a call 35; with more waves than
// the chip holds 45).
constexpr int kBackWaves = 8;  // waves of a workgroup of the backward pass

template <typename T, int DH, bool HALVES, bool VEC>
__global__ __launch_bounds__(64 * kBackWaves, VEC && sizeof(T) == 2 ? 3 : 2) void qk_rotate_back_kernel(const RopeArgs a) {
  constexpr int kLPH = DH / 8, kHPW = kWave / kLPH, kU = 2;
  __shared__ float red[kBackWaves][2][DH];
  const int lane = threadIdx.x % kWave, p0 = 4 * (lane % kLPH), sub = lane / kLPH;
  const int64_t wave = int64_t(blockIdx.x) * kBackWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // (row, part) pairs, a.per of them one after another to a wave.
  const int64_t first = wave * a.per, last = std::min(a.M * a.parts, first + a.per);
  typedef Lane<T, HALVES, VEC> At;
  const At at(p0, a.rot, sub * DH);
  const Turns<T> turns(a, p0);
  float acc[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[w][i] = 0.f;
  for (int64_t unit = first; unit < last; ++unit) {
    const int64_t row = unit / a.parts;
    const int part = int(unit % a.parts);
    const Span span[2] = {Span(a.H[0], kHPW, part, a.parts), Span(a.H[1], kHPW, part, a.parts)};
    typename At::Raw rx[2][kU], ry[2][kU];
    auto fetch = [&](int w, int st) {
      const T* in = static_cast<const T*>(a.x[w]) + row * a.x_ld[w];
      const T* dy = static_cast<const T*>(a.dy[w]) + row * a.dy_ld[w];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u < span[w].up && t < a.H[w]) {
          ry[w][u] = at.fetch(dy + (st + u) * (kHPW * DH));
          rx[w][u] = at.fetch(in + (st + u) * (kHPW * DH));
        }
      }
    };
#pragma unroll
    for (int w = 0; w < 2; ++w) fetch(w, span[w].lo);
    float s[4], c[4];
    turns.at(a, row, s, c);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = -s[i];  // back
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if (span[w].lo >= span[w].up) continue;
      float ga[4], gb[4];
      load_gain<T, DH>(at, sub * DH, a.g[w], ga, gb);
      T* out = static_cast<T*>(a.out[w]) + row * a.out_ld[w];
      for (int st = span[w].lo; st < span[w].up; st += kU) {
        if (st > span[w].lo) fetch(w, st);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int t = (st + u) * kHPW + sub;
          if (st + u >= span[w].up || t >= a.H[w]) continue;
          float va[4], vb[4], ea[4], eb[4];
          at.unpack(ry[w][u], ea, eb);
          at.unpack(rx[w][u], va, vb);
          turns.turn(ea, eb, s, c);
          if (a.eps > 0.f) {
            float sum = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += va[i] * va[i] + vb[i] * vb[i];
            const float r = rsqrtf(group_sum(sum, kLPH) * (1.f / DH) + a.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              va[i] *= r;
              vb[i] *= r;
              const float ta = ea[i] * va[i], tb = eb[i] * vb[i];
              acc[w][i] += ta;
              acc[w][4 + i] += tb;
              dot += ta * ga[i] + tb * gb[i];
            }
            dot = group_sum(dot, kLPH) * (1.f / DH);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              ea[i] = r * (ea[i] * ga[i] - va[i] * dot);
              eb[i] = r * (eb[i] * gb[i] - vb[i] * dot);
            }
          }
          at.store(out + (st + u) * (kHPW * DH), ea, eb);
        }
      }
    }
  }
  if (!a.part) return;
  // The heads of a wave, then the waves.
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = acc[w][i];
#pragma unroll
      for (int o = kLPH; o < kWave; o *= 2) v += __shfl_xor(v, o);
      if (sub == 0) {
        int e;
        if constexpr (VEC) e = HALVES ? (i < 4 ? at.a[0] + i : at.b[0] + i - 4) : 2 * (p0 + i % 4) + i / 4;
        else e = i < 4 ? at.a[i % 4] : at.b[i % 4];  // head 0's lanes: no offset
        red[threadIdx.x / kWave][w][e] = v;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * DH; i += 64 * kBackWaves) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kBackWaves; ++k) v += red[k][i / DH][i % DH];
    a.part[int64_t(blockIdx.x) * 2 * DH + i] = v;
  }
}

// The workgroups' sums added up: 32 columns, 32 strands of rows to a workgroup.  A launch's latency: 1.7 to 3.8 us.
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* part, int64_t n, int d, float* dgq, float* dgk) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x % 32, col = blockIdx.x * 32 + lane, strand = threadIdx.x / 32;
  float v = 0.f;
  for (int64_t i = strand; i < n; i += 32 * 8) {  // eight rows under way together
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = i + 32 * u < n ? part[(i + 32 * u) * 2 * d + col] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) v += x[u];
  }
  red[strand][lane] = v;
  __syncthreads();
  if (strand != 0) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) v += red[i][lane];
  float* dst = col < d ? dgq : dgk;
  if (dst) dst[col % d] = v;
}

// Forward: rows of a wave, and waves to a row where rows are few: about kForwardWaves waves (fewer where a wave would
// have no step of the queries or the keys).
constexpr int64_t kForwardWaves = 16384;
int most_parts(const RopeArgs& a, int d) {
  const int hpw = kWave / (d / 8);
  return (std::max(a.H[0], a.H[1]) + hpw - 1) / hpw;
}
void plan_forward(RopeArgs& a, int d) {
  a.per = std::max<int64_t>(1, a.M / kForwardWaves);
  const int64_t units = ceil_div64(a.M, a.per);
  a.parts = int(std::min<int64_t>(most_parts(a, d), std::max<int64_t>(1, (kForwardWaves + units / 2) / units)));
}
// Backward: each wave ends with a sum over its lanes and its workgroup's, so there are no more than the chip holds
// at once, with as many (row, part) pairs each; parts of two steps of the queries and two of the keys, which
// are under way together.
constexpr int64_t kBackwardWaves = 12 * 256;  // twelve to a CU
void plan_backward(RopeArgs& a, int d) {
  a.parts = std::max(1, most_parts(a, d) / 2);
  if (a.M * a.parts < kBackwardWaves) a.parts = int(std::min<int64_t>(most_parts(a, d), ceil_div64(kBackwardWaves, a.M)));
  a.per = ceil_div64(a.M * a.parts, kBackwardWaves);
}
int64_t back_workgroups(const RopeArgs& a) { return ceil_div64(ceil_div64(a.M * a.parts, a.per), kBackWaves); }

bool whole(const void* p, int64_t ld, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * int64_t(elem) % 16 == 0;
}

template <typename T, bool BACK, int DH, bool HALVES>
void launch_layout(const RopeArgs& a, bool vec, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(BACK ? back_workgroups(a) : ceil_div64(ceil_div64(a.M, a.per) * a.parts, 4)));
  const dim3 block(BACK ? 64 * kBackWaves : 256);
  if constexpr (BACK) {
    if (vec) hipLaunchKernelGGL((qk_rotate_back_kernel<T, DH, HALVES, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((qk_rotate_back_kernel<T, DH, HALVES, false>), grid, block, 0, s, a);
  } else {
    if (vec) hipLaunchKernelGGL((qk_rotate_kernel<T, DH, HALVES, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((qk_rotate_kernel<T, DH, HALVES, false>), grid, block, 0, s, a);
  }
}

template <typename T, bool BACK>
void launch_type(const RopeArgs& a, int d, bool halves, hipStream_t s) {
  bool vec = !halves || a.rot % 8 == 0;
  for (int w = 0; w < 2; ++w) {
    if (a.H[w] == 0) continue;
    vec = vec && whole(a.x[w], a.x_ld[w], sizeof(T)) && whole(a.out[w], a.out_ld[w], sizeof(T)) &&
          (!BACK || whole(a.dy[w], a.dy_ld[w], sizeof(T)));
  }
  if (d == 128) halves ? launch_layout<T, BACK, 128, true>(a, vec, s) : launch_layout<T, BACK, 128, false>(a, vec, s);
  else halves ? launch_layout<T, BACK, 64, true>(a, vec, s) : launch_layout<T, BACK, 64, false>(a, vec, s);
}

// Checks what both directions share and fills the arguments in.
int fill(RopeArgs& a, const char* what, const void* q, int64_t q_ld, const void* k, int64_t k_ld, int64_t M, int32_t H,
         int32_t Hk, int32_t d, const void* g_q, const void* g_k, float eps, const avits_rope* rope, int dtype, void* q_out,
         int64_t qo_ld, void* k_out, int64_t ko_ld) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 31), "%s: M=%lld outside [0, 2^31)", what, (long long)M);
  AVITS_REQUIRE(H >= 0 && Hk >= 0 && H + int64_t(Hk) >= 1 && H <= 1024 && Hk <= 1024,
                "%s: H=%d Hk=%d (0 to 1024 each, not both 0)", what, H, Hk);
  if (d != 64 && d != 128) return set_error(AVITS_ERR_UNSUPPORTED, "%s: head dim %d (need 64 or 128)", what, d);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", what, dtype);
  AVITS_REQUIRE(eps >= 0.f && eps < INFINITY, "%s: eps must be finite and >= 0", what);
  AVITS_REQUIRE(eps > 0.f || (!g_q && !g_k), "%s: a gain without a norm (eps 0)", what);
  AVITS_REQUIRE(M == 0 || ((H == 0 || (q && q_out)) && (Hk == 0 || (k && k_out))), "%s: null rows", what);
  const uintptr_t elem = dtype == AVITS_BF16 ? 2 : 4;
  for (const void* p : {q, k, static_cast<const void*>(q_out), static_cast<const void*>(k_out), g_q, g_k})
    AVITS_REQUIRE(reinterpret_cast<uintptr_t>(p) % elem == 0, "%s: a pointer is not aligned to its element", what);
  AVITS_REQUIRE(M <= 1 || ((H == 0 || (q_ld >= int64_t(H) * d && qo_ld >= int64_t(H) * d)) &&
                           (Hk == 0 || (k_ld >= int64_t(Hk) * d && ko_ld >= int64_t(Hk) * d))),
                "%s: rows overlap (row strides must be at least heads * d)", what);
  AVITS_REQUIRE(q_ld < (int64_t(1) << 31) && k_ld < (int64_t(1) << 31) && qo_ld < (int64_t(1) << 31) && ko_ld < (int64_t(1) << 31),
                "%s: row strides must be below 2^31", what);
  a = RopeArgs{};
  a.pos_scale = 1.0;
  if (rope) {
    AVITS_REQUIRE(rope->axes >= 1 && rope->axes <= kMaxAxes, "%s: axes=%d outside [1, %d]", what, rope->axes, kMaxAxes);
    AVITS_REQUIRE(rope->layout == AVITS_ROPE_PAIRS || rope->layout == AVITS_ROPE_HALVES, "%s: layout %d", what, rope->layout);
    int64_t rot = 0;
    for (int x = 0; x < rope->axes; ++x) {
      AVITS_REQUIRE(rope->dims[x] >= 0 && rope->dims[x] % 2 == 0 && rope->dims[x] <= d, "%s: dims[%d]=%d (even, at most d)", what, x, rope->dims[x]);
      rot += rope->dims[x];
      a.end[x] = int(rot / 2);
    }
    AVITS_REQUIRE(rot <= d, "%s: %lld rotated elements in a head of %d", what, (long long)rot, d);
    AVITS_REQUIRE(std::isfinite(rope->pos_scale), "%s: pos_scale must be finite", what);
    AVITS_REQUIRE(rot == 0 || M == 0 || (rope->pos && rope->freq), "%s: null pos or freq", what);
    AVITS_REQUIRE(reinterpret_cast<uintptr_t>(rope->pos) % 4 == 0 && reinterpret_cast<uintptr_t>(rope->freq) % 8 == 0,
                  "%s: pos or freq is not aligned to its element", what);
    a.rot = int(rot);
    a.axes = rope->axes;
    a.pos = rope->pos;
    a.freq = rope->freq;
    a.pos_scale = rope->pos_scale;
  }
  a.x[0] = q, a.x[1] = k;
  a.x_ld[0] = q_ld, a.x_ld[1] = k_ld;
  a.out[0] = q_out, a.out[1] = k_out;
  a.out_ld[0] = qo_ld, a.out_ld[1] = ko_ld;
  a.g[0] = g_q, a.g[1] = g_k;
  a.M = M;
  a.H[0] = H, a.H[1] = Hk;
  a.eps = eps;
  return AVITS_OK;
}

// Enough for the plan of any number of rows up to M.
size_t part_bytes(int64_t M, int32_t H, int32_t Hk, int32_t d) {
  RopeArgs a{};
  a.H[0] = H, a.H[1] = Hk;
  const int64_t waves = std::min<int64_t>(kBackwardWaves, std::max<int64_t>(M, 1) * most_parts(a, d));
  return size_t(ceil_div64(waves, kBackWaves)) * 2 * d * sizeof(float);
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" int avits_rope_frequencies(int32_t axes, const int32_t* dims, double theta, double factor, int64_t trained,
                                      double low, double high, double* freq) {
  AVITS_REQUIRE(axes >= 1 && axes <= kMaxAxes && dims && freq, "rope_frequencies: axes=%d outside [1, %d] or a null pointer", axes, kMaxAxes);
  AVITS_REQUIRE(theta > 0 && std::isfinite(theta) && factor > 0 && std::isfinite(factor), "rope_frequencies: theta and factor must be positive and finite");
  AVITS_REQUIRE(trained >= 0 && (trained == 0 || (low >= 0 && high > low && std::isfinite(high))),
                "rope_frequencies: trained=%lld must be >= 0, and 0 <= low < high where it is not 0", (long long)trained);
  for (int x = 0; x < axes; ++x)
    AVITS_REQUIRE(dims[x] >= 0 && dims[x] % 2 == 0 && dims[x] <= 1024, "rope_frequencies: dims[%d]=%d (even, 0 to 1024)", x, dims[x]);
  int at = 0;
  for (int x = 0; x < axes; ++x)
    for (int m = 0; m < dims[x] / 2; ++m) {
      const double f = pow(theta, -2.0 * m / dims[x]);
      double keep = 0.0;  // the share of the frequency that is not interpolated
      if (trained > 0) keep = std::min(1.0, std::max(0.0, (double(trained) * f * 0.15915494309189533577 - low) / (high - low)));
      freq[at++] = f * (keep + (1.0 - keep) / factor);
    }
  return AVITS_OK;
}

extern "C" int avits_qk_norm_rope(const void* q, int64_t q_ld, const void* k, int64_t k_ld, int64_t M, int32_t H, int32_t Hk,
                                  int32_t d, const void* g_q, const void* g_k, float eps, const avits_rope* rope, int dtype,
                                  void* q_out, int64_t qo_ld, void* k_out, int64_t ko_ld, void* stream) {
  RopeArgs a;
  const int rc = fill(a, "qk_norm_rope", q, q_ld, k, k_ld, M, H, Hk, d, g_q, g_k, eps, rope, dtype, q_out, qo_ld, k_out, ko_ld);
  if (rc != AVITS_OK || M == 0) return rc;
  plan_forward(a, d);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool halves = rope && rope->layout == AVITS_ROPE_HALVES;
  TimedLaunch timed("qk_norm_rope", s);
  if (dtype == AVITS_BF16) launch_type<bf16_t, false>(a, d, halves, s);
  else launch_type<float, false>(a, d, halves, s);
  return launch_status("qk_norm_rope");
}

extern "C" size_t avits_qk_norm_rope_backward_workspace_bytes(int64_t M, int32_t H, int32_t Hk, int32_t d) {
  if (M < 0 || M >= (int64_t(1) << 31) || H < 0 || Hk < 0 || H > 1024 || Hk > 1024 || H + Hk < 1 || (d != 64 && d != 128)) return 0;
  return part_bytes(M, H, Hk, d);
}

extern "C" int avits_qk_norm_rope_backward(const void* dq_out, int64_t dqo_ld, const void* dk_out, int64_t dko_ld, const void* q,
                                           int64_t q_ld, const void* k, int64_t k_ld, int64_t M, int32_t H, int32_t Hk, int32_t d,
                                           const void* g_q, const void* g_k, float eps, const avits_rope* rope, int dtype,
                                           void* dq, int64_t dq_ld, void* dk, int64_t dk_ld, float* dg_q, float* dg_k,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "qk_norm_rope_backward";
  RopeArgs a;
  // Without a norm the rows themselves are not needed.
  const bool norm = eps > 0.f;
  int rc = fill(a, what, norm ? q : dq_out, norm ? q_ld : dqo_ld, norm ? k : dk_out, norm ? k_ld : dko_ld, M, H, Hk, d, g_q, g_k, eps,
                rope, dtype, dq, dq_ld, dk, dk_ld);
  if (rc != AVITS_OK) return rc;
  const uintptr_t elem = dtype == AVITS_BF16 ? 2 : 4;
  AVITS_REQUIRE(M == 0 || ((H == 0 || dq_out) && (Hk == 0 || dk_out)), "%s: null gradients", what);
  AVITS_REQUIRE(reinterpret_cast<uintptr_t>(dq_out) % elem == 0 && reinterpret_cast<uintptr_t>(dk_out) % elem == 0 &&
                    reinterpret_cast<uintptr_t>(dg_q) % 4 == 0 && reinterpret_cast<uintptr_t>(dg_k) % 4 == 0,
                "%s: a pointer is not aligned to its element", what);
  AVITS_REQUIRE(M <= 1 || ((H == 0 || dqo_ld >= int64_t(H) * d) && (Hk == 0 || dko_ld >= int64_t(Hk) * d)),
                "%s: rows overlap (row strides must be at least heads * d)", what);
  AVITS_REQUIRE(dqo_ld < (int64_t(1) << 31) && dko_ld < (int64_t(1) << 31), "%s: row strides must be below 2^31", what);
  AVITS_REQUIRE(norm || (!dg_q && !dg_k), "%s: a gain's gradient without a norm (eps 0)", what);
  AVITS_REQUIRE((!dg_q || H > 0) && (!dg_k || Hk > 0), "%s: a gain's gradient without heads", what);
  a.dy[0] = dq_out, a.dy[1] = dk_out;
  a.dy_ld[0] = dqo_ld, a.dy_ld[1] = dko_ld;
  const bool sums = dg_q || dg_k;
  if (sums) {
    const size_t need = part_bytes(M, H, Hk, d);
    if (!workspace || workspace_bytes < need)
      return set_error(AVITS_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : size_t(0), need);
    AVITS_REQUIRE(reinterpret_cast<uintptr_t>(workspace) % 16 == 0, "%s: the workspace is not 16-byte aligned", what);
    a.part = static_cast<float*>(workspace);
  }
  if (M == 0 && !sums) return AVITS_OK;
  if (M > 0) plan_backward(a, d);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool halves = rope && rope->layout == AVITS_ROPE_HALVES;
  TimedLaunch timed(what, s);
  const int64_t n = M == 0 ? 0 : back_workgroups(a);
  if (M > 0) {
    if (dtype == AVITS_BF16) launch_type<bf16_t, true>(a, d, halves, s);
    else launch_type<float, true>(a, d, halves, s);
  }
  if (sums) hipLaunchKernelGGL(gain_sum_kernel, dim3(2 * d / 32), dim3(1024), 0, s, a.part, n, d, dg_q, dg_k);
  return launch_status(what);
}
