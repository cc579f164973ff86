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
  int a[VEC ? 1 : 4], b[VEC ? 1 : 4];
  __device__ __forceinline__ Lane(int p0, int rot) {
    if constexpr (VEC) {
      a[0] = 2 * p0;
      b[0] = 2 * p0 + 4;
      if (HALVES && p0 < rot / 2) {
        a[0] = p0;
        b[0] = p0 + rot / 2;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i;
        const bool split = HALVES && p < rot / 2;
        a[i] = split ? p : 2 * p;
        b[i] = split ? p + rot / 2 : 2 * p + 1;
      }
    }
  }
  __device__ __forceinline__ static void four(const T* p, float* v) {
    if constexpr (sizeof(T) == 4) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = w[i];
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ static void put4(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    else *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
  }
  // The first and the second elements of the four pairs.
  __device__ __forceinline__ void load(const T* p, float* va, float* vb) const {
    if constexpr (VEC) {
      if constexpr (HALVES) {
        four(p + a[0], va);
        four(p + b[0], vb);
      } else {
        float v[8];
        if constexpr (sizeof(T) == 4) {
          four(p + a[0], v);
          four(p + a[0] + 4, v + 4);
        } else {
          const u32x4 w = *reinterpret_cast<const u32x4*>(p + a[0]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          va[i] = v[2 * i];
          vb[i] = v[2 * i + 1];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        va[i] = ld(p, a[i]);
        vb[i] = ld(p, b[i]);
      }
    }
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

// The turns of a row's four pairs of this lane (pairs past rot: none).
template <typename T>
struct Turns {
  double f[4];
  int axis[4];
  __device__ __forceinline__ Turns(const RopeArgs& a, int p0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + i;
      axis[i] = -1;
      f[i] = 0.0;
      if (2 * p < a.rot) {
        f[i] = a.freq[p];
        axis[i] = 0;
#pragma unroll
        for (int x = 0; x < kMaxAxes - 1; ++x) axis[i] += x < a.axes - 1 && p >= a.end[x] ? 1 : 0;
      }
    }
  }
  __device__ __forceinline__ void at(const RopeArgs& a, int64_t row, float* s, float* c) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = 0.f;
      c[i] = 1.f;
      if (axis[i] >= 0) {
        const double turns = double(a.pos[row * a.axes + axis[i]]) * a.pos_scale * f[i] * 0.15915494309189533577;
        turn_of<T>(float(turns - rint(turns)), s[i], c[i]);
      }
    }
  }
};

template <typename T, int DH, bool HALVES, bool VEC>
__global__ __launch_bounds__(256) void qk_rotate_kernel(const RopeArgs a) {
  constexpr int kLPH = DH / 8, kHPW = kWave / kLPH, kU = 4;  // lanes to a head, heads to a step, steps at once
  const int lane = threadIdx.x % kWave, p0 = 4 * (lane % kLPH), sub = lane / kLPH;
  const int64_t wave = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave;
  const int part = int(wave % a.parts);
  const int64_t first = wave / a.parts * a.per, last = std::min(a.M, first + a.per);
  const int heads = a.H[0] + a.H[1], steps = (heads + kHPW - 1) / kHPW;
  const int s_lo = steps * part / a.parts, s_hi = steps * (part + 1) / a.parts;
  if (first >= last) return;
  const Lane<T, HALVES, VEC> at(p0, a.rot);
  const Turns<T> turns(a, p0);
  float g[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[w][i] = 1.f;
    if (a.g[w]) {
      const Lane<T, HALVES, false> one(p0, a.rot);
      const T* gw = static_cast<const T*>(a.g[w]);
      if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[w][i] = ld(gw, HALVES ? at.a[0] + i : 2 * (p0 + i));
          g[w][4 + i] = ld(gw, HALVES ? at.b[0] + i : 2 * (p0 + i) + 1);
        }
      } else {
        one.load(gw, g[w], g[w] + 4);
      }
    }
  }
  for (int64_t row = first; row < last; ++row) {
    float s[4], c[4];
    turns.at(a, row, s, c);
    for (int st = s_lo; st < s_hi; st += kU) {
      float va[kU][4], vb[kU][4];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u < s_hi && t < heads) {
          const int w = t >= a.H[0];
          const T* p = static_cast<const T*>(w ? a.x[1] : a.x[0]) + row * (w ? a.x_ld[1] : a.x_ld[0]) +
                       int64_t(w ? t - a.H[0] : t) * DH;
          at.load(p, va[u], vb[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u >= s_hi || t >= heads) continue;
        const int w = t >= a.H[0];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += va[u][i] * va[u][i] + vb[u][i] * vb[u][i];
        sum = group_sum(sum, kLPH);
        const float r = a.eps > 0.f ? rsqrtf(sum * (1.f / DH) + a.eps) : 1.f;
        float oa[4], ob[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ya = va[u][i] * r * (w ? g[1][i] : g[0][i]), yb = vb[u][i] * r * (w ? g[1][4 + i] : g[0][4 + i]);
          // Elements that do not turn are no pair: what one holds is not the other's.
          const bool on = turns.axis[i] >= 0;
          oa[i] = on ? ya * c[i] - yb * s[i] : ya;
          ob[i] = on ? ya * s[i] + yb * c[i] : yb;
        }
        T* p = static_cast<T*>(w ? a.out[1] : a.out[0]) + row * (w ? a.out_ld[1] : a.out_ld[0]) +
               int64_t(w ? t - a.H[0] : t) * DH;
        at.store(p, oa, ob);
      }
    }
  }
}

template <typename T, int DH, bool HALVES, bool VEC>
__global__ __launch_bounds__(256) void qk_rotate_back_kernel(const RopeArgs a) {
  constexpr int kLPH = DH / 8, kHPW = kWave / kLPH, kU = 2;
  __shared__ float red[4][2][DH];
  const int lane = threadIdx.x % kWave, p0 = 4 * (lane % kLPH), sub = lane / kLPH;
  const int64_t wave = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave;
  const int part = int(wave % a.parts);
  const int64_t first = wave / a.parts * a.per, last = std::min(a.M, first + a.per);
  const int heads = a.H[0] + a.H[1], steps = (heads + kHPW - 1) / kHPW;
  const int s_lo = steps * part / a.parts, s_hi = steps * (part + 1) / a.parts;
  const Lane<T, HALVES, VEC> at(p0, a.rot);
  const Turns<T> turns(a, p0);
  float g[2][8], acc[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[w][i] = 1.f, acc[w][i] = 0.f;
    if (a.g[w]) {
      const T* gw = static_cast<const T*>(a.g[w]);
      if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[w][i] = ld(gw, HALVES ? at.a[0] + i : 2 * (p0 + i));
          g[w][4 + i] = ld(gw, HALVES ? at.b[0] + i : 2 * (p0 + i) + 1);
        }
      } else {
        at.load(gw, g[w], g[w] + 4);
      }
    }
  }
  for (int64_t row = first; row < last; ++row) {
    float s[4], c[4];
    turns.at(a, row, s, c);
    for (int st = s_lo; st < s_hi; st += kU) {
      float va[kU][4], vb[kU][4], ea[kU][4], eb[kU][4];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u < s_hi && t < heads) {
          const int w = t >= a.H[0];
          const int64_t col = int64_t(w ? t - a.H[0] : t) * DH;
          at.load(static_cast<const T*>(w ? a.x[1] : a.x[0]) + row * (w ? a.x_ld[1] : a.x_ld[0]) + col, va[u], vb[u]);
          at.load(static_cast<const T*>(w ? a.dy[1] : a.dy[0]) + row * (w ? a.dy_ld[1] : a.dy_ld[0]) + col, ea[u], eb[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int t = (st + u) * kHPW + sub;
        if (st + u >= s_hi || t >= heads) continue;
        const int w = t >= a.H[0];
        // The gradient turned back.
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float da = ea[u][i] * c[i] + eb[u][i] * s[i], db = eb[u][i] * c[i] - ea[u][i] * s[i];
          const bool on = turns.axis[i] >= 0;
          ea[u][i] = on ? da : ea[u][i];
          eb[u][i] = on ? db : eb[u][i];
        }
        if (a.eps > 0.f) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += va[u][i] * va[u][i] + vb[u][i] * vb[u][i];
          const float r = rsqrtf(group_sum(sum, kLPH) * (1.f / DH) + a.eps);
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float na = va[u][i] * r, nb = vb[u][i] * r;
            const float ta = ea[u][i] * na, tb = eb[u][i] * nb;
            acc[0][i] += w ? 0.f : ta;
            acc[0][4 + i] += w ? 0.f : tb;
            acc[1][i] += w ? ta : 0.f;
            acc[1][4 + i] += w ? tb : 0.f;
            const float ga = w ? g[1][i] : g[0][i], gb = w ? g[1][4 + i] : g[0][4 + i];
            ea[u][i] *= ga;
            eb[u][i] *= gb;
            dot += ta * ga + tb * gb;
            va[u][i] = na;
            vb[u][i] = nb;
          }
          dot = group_sum(dot, kLPH) * (1.f / DH);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ea[u][i] = r * (ea[u][i] - va[u][i] * dot);
            eb[u][i] = r * (eb[u][i] - vb[u][i] * dot);
          }
        }
        T* p = static_cast<T*>(w ? a.out[1] : a.out[0]) + row * (w ? a.out_ld[1] : a.out_ld[0]) +
               int64_t(w ? t - a.H[0] : t) * DH;
        at.store(p, ea[u], eb[u]);
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
        else e = i < 4 ? at.a[i % 4] : at.b[i % 4];
        red[threadIdx.x / kWave][w][e] = v;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * DH; i += 256) {
    const float* r = &red[0][0][0] + i;
    a.part[int64_t(blockIdx.x) * 2 * DH + i] = (r[0] + r[2 * DH]) + (r[4 * DH] + r[6 * DH]);
  }
}

// The workgroups' sums added up: 32 columns, eight strands of rows to a workgroup.
__global__ __launch_bounds__(256) void gain_sum_kernel(const float* part, int64_t n, int d, float* dgq, float* dgk) {
  __shared__ float red[8][32];
  const int col = blockIdx.x * 32 + threadIdx.x % 32, strand = threadIdx.x / 32;
  float v = 0.f;
#pragma unroll 8
  for (int64_t i = strand; i < n; i += 8) v += part[i * 2 * d + col];
  red[strand][threadIdx.x % 32] = v;
  __syncthreads();
  if (strand != 0) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) v += red[i][threadIdx.x];
  float* dst = col < d ? dgq : dgk;
  if (dst) dst[col % d] = v;
}

// Rows of a wave and waves to a row: enough waves for every SIMD of the chip
// to hold several, then as many heads to a wave as that leaves.
void plan(RopeArgs& a, int d, int64_t waves) {
  const int hpw = kWave / (d / 8), steps = (a.H[0] + a.H[1] + hpw - 1) / hpw;
  a.per = std::max<int64_t>(1, ceil_div64(a.M, waves));
  a.parts = int(std::min<int64_t>(steps, std::max<int64_t>(1, waves / ceil_div64(a.M, a.per))));
}
constexpr int64_t kForwardWaves = 16384, kBackwardWaves = 2048;

int64_t workgroups(const RopeArgs& a) { return ceil_div64(ceil_div64(a.M, a.per) * a.parts, 4); }

bool whole(const void* p, int64_t ld, size_t elem) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * int64_t(elem) % 16 == 0;
}

template <typename T, bool BACK, int DH, bool HALVES>
void launch_layout(const RopeArgs& a, bool vec, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(workgroups(a))), block(256);
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
  const int hpw = kWave / (d / 8), steps = (H + Hk + hpw - 1) / hpw;
  const int64_t wgs = ceil_div64(std::min<int64_t>(kBackwardWaves, std::max<int64_t>(M, 1) * steps), 4);
  return size_t(wgs) * 2 * d * sizeof(float);
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
  plan(a, d, kForwardWaves);
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
  if (M > 0) plan(a, d, kBackwardWaves);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool halves = rope && rope->layout == AVITS_ROPE_HALVES;
  TimedLaunch timed(what, s);
  const int64_t n = M == 0 ? 0 : workgroups(a);
  if (M > 0) {
    if (dtype == AVITS_BF16) launch_type<bf16_t, true>(a, d, halves, s);
    else launch_type<float, true>(a, d, halves, s);
  }
  if (sums) hipLaunchKernelGGL(gain_sum_kernel, dim3(2 * d / 32), dim3(256), 0, s, a.part, n, d, dg_q, dg_k);
  return launch_status(what);
}
