// The modulated layer norm with its statistics, and its backward pass.
//
//   n = (x - mean) rstd,   h = n (1 + scale) + shift
//   g = dh (1 + scale),    dx = rstd (g - avg(g) - n avg(g n)) [+ dres]
//   dscale = sum over rows of dh n,   dshift = sum over rows of dh
//
// Rows of several images lie one after another; image b's rows take the
// vectors b * mod_stride elements after the first image's.
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "lowbit.h"

namespace avits {
namespace {

template <typename T>
__device__ __forceinline__ float one_or(const T* p, int64_t i) { return p ? 1.f + ld(p, i) : 1.f; }

// Rows that are shorter than 16 bytes or longer than registers hold: a wave per
// row, elements one by one, the row read three times (it stays in the caches).
template <typename T>
__global__ __launch_bounds__(256) void norm_any_kernel(const T* x, int64_t M, int64_t D, const Images im,
                                                       const T* __restrict__ shift, const T* __restrict__ scale,
                                                       float eps, T* h, float* __restrict__ mean, float* __restrict__ rstd) {
  const int lane = threadIdx.x % kWave;
  const int64_t row = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave;
  if (row >= M) return;
  const T* xr = x + row * D;
  float s = 0.f;
  for (int64_t i = lane; i < D; i += kWave) s += ld(xr, i);
  const float mu = wave_sum(s) / float(D);
  float q = 0.f;
  for (int64_t i = lane; i < D; i += kWave) {
    const float d = ld(xr, i) - mu;
    q = fmaf(d, d, q);
  }
  const float rs = rsqrtf(wave_sum(q) / float(D) + eps);
  const int64_t mo = int64_t(image_of(im, row)) * im.stride;
  for (int64_t i = lane; i < D; i += kWave)
    st(h, row * D + i, (ld(xr, i) - mu) * rs * one_or(scale, mo + i) + (shift ? ld(shift, mo + i) : 0.f));
  if (lane == 0) {
    if (mean) mean[row] = mu;
    if (rstd) rstd[row] = rs;
  }
}

// 16 bytes of a row as floats, and back.
template <typename T> constexpr int kVec = 16 / int(sizeof(T));
template <typename T>
__device__ __forceinline__ void widen(const u32x4& w, float (&v)[kVec<T>]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    } else {
      v[e] = __uint_as_float(w[e]);
    }
  }
}
template <typename T>
__device__ __forceinline__ u32x4 narrow(const float (&v)[kVec<T>]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) w[e] = pack_bf2(v[2 * e], v[2 * e + 1]);
    else w[e] = __float_as_uint(v[e]);
  }
  return w;
}

// A row's chunks of 16 bytes, at any element.  TAIL: its last chunk is partial and
// taken from the row's end; its first `dup` elements belong to the chunk before
// it, whose lane gives them the same bits, and are left out of sums over the row.
template <int E, bool TAIL>
struct ChunkAt {
  int pos, dup;
  __device__ __forceinline__ ChunkAt(int at, int D) : pos(E * at), dup(0) {
    if (TAIL && pos + E > D) {
      dup = pos + E - D;
      pos = D - E;
    }
  }
};
// (Under a branch that one wave of a row takes.)
template <int E>
__device__ __forceinline__ void zero_first(float (&v)[E], int n) {
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = e < n ? 0.f : v[e];
}
template <typename T>
__device__ __forceinline__ u32x4 chunk_of(const T* p) {
  const loose4 w = *reinterpret_cast<const loose4*>(p);
  return u32x4{w[0], w[1], w[2], w[3]};
}
template <typename T>
__device__ __forceinline__ void put_chunk(T* p, const u32x4& w) {
  *reinterpret_cast<loose4*>(p) = loose4{w[0], w[1], w[2], w[3]};
}

// WAVES waves hold a row in registers, NC chunks in a lane (chunk l + 64 WAVES c), so
// memory is read once and written once, which is the bound.  A workgroup takes
// `per` consecutive rows, keeps the modulation of an image as long as its rows
// last, and loads the next row while it reduces one.  (h may be x: a row's sums
// need all of it, so its loads are done before its first store.)  Measured (its bytes
// at a large copy's rate in brackets): 16000 x 2048 bf16 27.5 us (25.7), x 3999
// 57.7 (50.2; element by element, reading rows again, 235), x 8192 fp32 212 (206).
template <typename T, int NC, int WAVES, bool TAIL>
__global__ __launch_bounds__(256) void norm_rows_kernel(const T* x, int64_t M, int64_t D, const Images im,
                                                        const T* __restrict__ shift, const T* __restrict__ scale, float eps,
                                                        T* h, float* __restrict__ mean, float* __restrict__ rstd, int per) {
  constexpr int E = kVec<T>, kTeams = 4 / WAVES;
  __shared__ float red[2][4];
  const int lane = threadIdx.x % (kWave * WAVES), team = threadIdx.x / (kWave * WAVES);
  const int width = int(D), nchunk = (width + E - 1) / E;
  const int64_t first = (int64_t(blockIdx.x) * kTeams + team) * per, last = std::min<int64_t>(first + per, M);
  const float inv = 1.f / float(D);
  auto load = [&](int64_t row, u32x4 (&v)[NC]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = lane + kWave * WAVES * c;
      v[c] = at < nchunk ? chunk_of(x + row * D + ChunkAt<E, TAIL>(at, width).pos) : u32x4{0u, 0u, 0u, 0u};
    }
  };
  auto total = [&](float s, int slot) {
    s = wave_sum(s);
    if constexpr (WAVES > 1) {
      if (threadIdx.x % kWave == 0) red[slot][threadIdx.x / kWave] = s;
      __syncthreads();
      s = (red[slot][0] + red[slot][1]) + (red[slot][2] + red[slot][3]);
    }
    return s;
  };
  u32x4 cur[NC], nxt[NC], g[NC], t[NC];
  int image = -1;
  if (first < last) load(first, cur);
  for (int64_t row = first; row < last; ++row) {
    if (row + 1 < last) load(row + 1, nxt);
    const int b = image_of(im, row);
    if (b != image) {
      image = b;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int at = lane + kWave * WAVES * c, pos = ChunkAt<E, TAIL>(at, width).pos;
        g[c] = scale && at < nchunk ? chunk_of(scale + b * im.stride + pos) : u32x4{0u, 0u, 0u, 0u};
        t[c] = shift && at < nchunk ? chunk_of(shift + b * im.stride + pos) : u32x4{0u, 0u, 0u, 0u};
      }
    }
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[E];
      widen<T>(cur[c], v);
      const ChunkAt<E, TAIL> here(lane + kWave * WAVES * c, width);
      if (TAIL && here.dup > 0) zero_first(v, here.dup);
#pragma unroll
      for (int e = 0; e < E; e += 2) s += v[e] + v[e + 1];
    }
    const float mu = total(s, 0) * inv;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[E];
      widen<T>(cur[c], v);
      const int at = lane + kWave * WAVES * c;
      const ChunkAt<E, TAIL> here(at, width);
      if (at < nchunk) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] -= mu;
        if (TAIL && here.dup > 0) zero_first(v, here.dup);
#pragma unroll
        for (int e = 0; e < E; ++e) q = fmaf(v[e], v[e], q);
      }
    }
    const float rs = rsqrtf(total(q, 1) * inv + eps);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = lane + kWave * WAVES * c;
      if (at < nchunk) {
        float v[E], w[E], z[E];
        widen<T>(cur[c], v);
        widen<T>(g[c], w);
        widen<T>(t[c], z);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (v[e] - mu) * rs * (1.f + w[e]) + z[e];
        put_chunk(h + row * D + ChunkAt<E, TAIL>(at, width).pos, narrow<T>(v));
      }
    }
    if (lane == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = rs;
    }
    if constexpr (WAVES > 1) __syncthreads();   // before the next row's sums
#pragma unroll
    for (int c = 0; c < NC; ++c) cur[c] = nxt[c];
  }
}

// Rows held in their own type or as 8-bit codes with scales.
template <typename T>
struct Rows {
  const T* x;
  const uint8_t* q;
  const uint8_t* s;
  int64_t ns;  // scales per row
};
template <typename T>
__device__ __forceinline__ float row_value(const Rows<T>& r, int64_t row, int64_t D, int64_t i) {
  if (r.x) return ld(r.x, row * D + i);
  return decode8(r.q[row * D + i], scale_value(r.s[row * r.ns + i / kBlk]));
}

// Where the column sums of the chunks go: chunk c's at scale + c stride, shift + c
// stride (each may be null).
struct SumsOut {
  float *scale, *shift;
  int64_t stride;
};

// Row chunks: chunk c covers rows [lo, hi) of one image; every image has at
// least one, so that an image without rows gets zero sums.
struct Chunks {
  int32_t first[kMaxSeqs + 1];  // chunk index of each image's first
  int32_t rows;                 // rows per chunk
};
__device__ __forceinline__ void chunk_rows(const Images& im, const Chunks& ch, int c, int& b, int64_t& lo, int64_t& hi) {
  b = 0;
#pragma unroll
  for (int i = 1; i < kMaxSeqs; ++i) b += (i < im.B && c >= ch.first[i]) ? 1 : 0;
  int64_t start = 0, end = im.end[0];
  int f = 0;
#pragma unroll
  for (int i = 1; i < kMaxSeqs; ++i)
    if (i <= b) {
      start = im.end[i - 1];
      end = im.end[i];
      f = ch.first[i];
    }
  lo = std::min<int64_t>(start + int64_t(c - f) * ch.rows, end);
  hi = std::min<int64_t>(lo + ch.rows, end);
}

// Backward of rows that are too short or too long for the kernel below, in two steps: the two averages of each row
// (a wave per row) ...
template <typename T>
__global__ __launch_bounds__(256) void norm_back_avg_kernel(const T* dh, const Rows<T> xr, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, int64_t M, int64_t D,
                                                            const Images im, const T* __restrict__ scale,
                                                            float* __restrict__ avg) {
  const int lane = threadIdx.x % kWave;
  const int64_t row = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave;
  if (row >= M) return;
  const int64_t mo = int64_t(image_of(im, row)) * im.stride;
  const float mu = mean[row], rs = rstd[row];
  float a = 0.f, b = 0.f;
  for (int64_t i = lane; i < D; i += kWave) {
    const float g = ld(dh, row * D + i) * one_or(scale, mo + i);
    a += g;
    b = fmaf(g, (row_value(xr, row, D, i) - mu) * rs, b);
  }
  a = wave_sum(a) / float(D);
  b = wave_sum(b) / float(D);
  if (lane == 0) {
    avg[2 * row] = a;
    avg[2 * row + 1] = b;
  }
}

// ... then a thread per column and chunk of rows: dx, and the chunk's sums.
template <typename T>
__global__ __launch_bounds__(256) void norm_back_any_kernel(const T* dh, const Rows<T> xr, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, int64_t D, const Images im,
                                                            const Chunks ch, const T* __restrict__ scale, const T* dres,
                                                            const float* __restrict__ avg, T* dx, const SumsOut sums) {
  const int c = blockIdx.x;
  const int64_t i = int64_t(blockIdx.y) * 256 + threadIdx.x;
  if (i >= D) return;
  int b;
  int64_t lo, hi;
  chunk_rows(im, ch, c, b, lo, hi);
  const float w = one_or(scale, int64_t(b) * im.stride + i);
  float sc = 0.f, sh = 0.f;
  for (int64_t row = lo; row < hi; ++row) {
    const float d = ld(dh, row * D + i), rs = rstd[row];
    const float n = (row_value(xr, row, D, i) - mean[row]) * rs;
    const float v = rs * (d * w - avg[2 * row] - n * avg[2 * row + 1]);
    st(dx, row * D + i, dres ? v + ld(dres, row * D + i) : v);
    sc = fmaf(d, n, sc);
    sh += d;
  }
  if (sums.scale) sums.scale[c * sums.stride + i] = sc;
  if (sums.shift) sums.shift[c * sums.stride + i] = sh;
}

// Backward: a workgroup takes a chunk of rows, R at a time; a thread owns NC
// vectors of columns for all of them, holds their weight and their column sums
// in registers, and the rows' two averages meet in LDS with one barrier for R
// rows.  Everything is read once and written once.  (dx may be dh or dres: rows are
// loaded whole before the barrier, so also where two lanes store the same elements.)
// Measured with the sums of the chunks: 16000 x 2048 bf16 48.0 us (38.6 at a copy's
// rate), from 8 bits 46.5 (32.1), x 3999 90.7 (75.3), x 8192 fp32 311 (308).
// Four vectors of bf16 columns to a thread (8193 to 16384 columns) leave no registers for
// the next rows nor for widened weights: there a row is loaded when its turn comes and
// what can be made again is.  8000 x 8200 117 us, from 8 bits 121, x 12001 194 and 192, x
// 16384 177 and 165 (with 40 to 174 registers in memory, as the form of fewer columns has it
// there: 285 and 230, 733 and 948, 408 and 354).
template <typename T, bool HELD, int NC, int R, bool TAIL>
__global__ __launch_bounds__(512) void norm_back_rows_kernel(const T* dh, const Rows<T> xr, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, int64_t D, const Images im,
                                                             const Chunks ch, const T* __restrict__ scale, const T* dres,
                                                             T* dx, const SumsOut sums) {
  constexpr int E = kVec<T>;
  constexpr bool kLean = NC == 4 && E == 8;
  __shared__ float red[2][8][2 * R];
  const int waves = blockDim.x / kWave, wave = threadIdx.x / kWave;
  const int width = int(D), nchunk = (width + E - 1) / E;
  const float inv = 1.f / float(D);
  int b;
  int64_t lo, hi;
  chunk_rows(im, ch, blockIdx.x, b, lo, hi);
  int at[NC], pos[NC], dup[NC];
  float w[kLean ? 1 : NC][E], sc[NC][E], sh[NC][E];
  u32x4 w_held[kLean ? NC : 1];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    at[c] = threadIdx.x + blockDim.x * c;
    const ChunkAt<E, TAIL> here(at[c], width);
    pos[c] = here.pos;
    dup[c] = here.dup;
    u32x4 g = {0u, 0u, 0u, 0u};
    if (scale && at[c] < nchunk) g = chunk_of(scale + b * im.stride + pos[c]);
    if constexpr (kLean) w_held[c] = g;
    else widen<T>(g, w[c]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (!kLean) w[c][e] = at[c] < nchunk ? 1.f + w[c][e] : 0.f;
      sc[c][e] = sh[c][e] = 0.f;
    }
  }
  auto weight = [&](int c, float (&v)[E]) {   // (past D dh is 0)
    if constexpr (kLean) {
      asm volatile("" : "+v"(w_held[c]));   // (opaque, here and below: what is widened is not kept)
      widen<T>(w_held[c], v);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (kLean) v[e] += 1.f;
      else v[e] = w[c][e];
    }
  };
  // The rows' data as loaded; rows past the chunk and columns past D as zeros.
  struct Batch {
    u32x4 d[R][NC], x[R][NC], r[R][NC];
    uint32_t s[R][NC], s_first[R][NC];   // (s_first: of a partial chunk's first elements, which may be of the block before)
    float mu[R], rs[R];
  };
  auto load = [&](int64_t row, Batch& t) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool in = row + r < hi;
      const int64_t m = in ? row + r : hi - 1;
      t.mu[r] = mean[m];
      t.rs[r] = rstd[m];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const bool here = in && at[c] < nchunk;
        if (kLean) asm volatile("" : "+v"(pos[c]));   // (nor are addresses)
        t.d[r][c] = here ? chunk_of(dh + m * D + pos[c]) : zero;
        t.x[r][c] = zero;
        if constexpr (HELD) {
          const uint8_t* q = xr.q + m * D + pos[c];
          if (here) {
            if constexpr (E == 8) {
              const loose2 v = *reinterpret_cast<const loose2*>(q);
              t.x[r][c][0] = v[0];
              t.x[r][c][1] = v[1];
            } else {
              t.x[r][c][0] = *reinterpret_cast<const loose1*>(q);
            }
          }
          t.s[r][c] = here ? xr.s[m * xr.ns + at[c] * E / kBlk] : 0u;
          if (TAIL) t.s_first[r][c] = here && dup[c] > 0 ? xr.s[m * xr.ns + pos[c] / kBlk] : 0u;
        } else if (here) {
          t.x[r][c] = chunk_of(xr.x + m * D + pos[c]);
        }
        t.r[r][c] = here && dres ? chunk_of(dres + m * D + pos[c]) : zero;
      }
    }
  };
  Batch t, next;
  if (!kLean && lo < hi) load(lo, t);
  int turn = 0;
  for (int64_t row = lo; row < hi; row += R, turn ^= 1) {
    if (kLean) load(row, t);
    else if (row + R < hi) load(row + R, next);
    auto normed = [&](int r, int c, float (&n)[E]) {
      if constexpr (HELD) {
        const float scale8 = scale_value(t.s[r][c]);
        decode8x4(t.x[r][c][0], scale8, n);
        if constexpr (E == 8) decode8x4(t.x[r][c][1], scale8, n + 4);
        if (TAIL && dup[c] > 0) {
          float first[E];
          decode8x4(t.x[r][c][0], scale_value(t.s_first[r][c]), first);
          if constexpr (E == 8) decode8x4(t.x[r][c][1], scale_value(t.s_first[r][c]), first + 4);
#pragma unroll
          for (int e = 0; e < E; ++e) n[e] = e < dup[c] ? first[e] : n[e];
        }
      } else {
        widen<T>(t.x[r][c], n);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) n[e] = (n[e] - t.mu[r]) * t.rs[r];
    };
    float sum[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[2 * r] = sum[2 * r + 1] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float dv[E], n[E], wv[E];
        widen<T>(t.d[r][c], dv);
        normed(r, c, n);
        weight(c, wv);
        if (TAIL && dup[c] > 0) {
          zero_first(dv, dup[c]);
          zero_first(n, dup[c]);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float g = dv[e] * wv[e];
          sum[2 * r] += g;
          sum[2 * r + 1] = fmaf(g, n[e], sum[2 * r + 1]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 2 * R; ++k) sum[k] = wave_sum(sum[k]);
    if (waves > 1) {
      if (threadIdx.x % kWave == 0)
#pragma unroll
        for (int k = 0; k < 2 * R; ++k) red[turn][wave][k] = sum[k];
      if constexpr (TAIL) {
        // dres too has arrived before another wave may store over its elements.
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int c = 0; c < NC; ++c) asm volatile("" ::"v"(t.r[r][c]) : "memory");
      }
      __syncthreads();   // the other half of red is read before the next one's barrier
#pragma unroll
      for (int k = 0; k < 2 * R; ++k) sum[k] = red[turn][0][k];
      for (int v = 1; v < waves; ++v)
#pragma unroll
        for (int k = 0; k < 2 * R; ++k) sum[k] += red[turn][v][k];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= hi) continue;
      const float ag = sum[2 * r] * inv, an = sum[2 * r + 1] * inv;
      if constexpr (kLean) {
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(t.d[r][c]), "+v"(t.x[r][c]));
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (at[c] >= nchunk) continue;
        float dv[E], n[E], o[E], wv[E];
        widen<T>(t.d[r][c], dv);
        normed(r, c, n);
        weight(c, wv);
        widen<T>(t.r[r][c], o);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          sc[c][e] = fmaf(dv[e], n[e], sc[c][e]);
          sh[c][e] += dv[e];
          o[e] += t.rs[r] * (dv[e] * wv[e] - ag - n[e] * an);
        }
        put_chunk(dx + (row + r) * D + pos[c], narrow<T>(o));
      }
    }
    if (!kLean) t = next;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (at[c] >= nchunk) continue;
    const int64_t o = blockIdx.x * sums.stride + pos[c];
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      if (sums.scale)
        put_chunk(sums.scale + o + e, __builtin_bit_cast(u32x4, f32x4{sc[c][e], sc[c][e + 1], sc[c][e + 2], sc[c][e + 3]}));
      if (sums.shift)
        put_chunk(sums.shift + o + e, __builtin_bit_cast(u32x4, f32x4{sh[c][e], sh[c][e + 1], sh[c][e + 2], sh[c][e + 3]}));
    }
  }
}

// Sums of the chunks' parts, in chunk order within each of 64 strands: 16 V
// columns of a workgroup (V = 4 where rows of D floats are aligned), blockIdx.y
// the image (or all of them together), blockIdx.z scale or shift.
template <int V>
__global__ __launch_bounds__(1024) void norm_back_sum_kernel(const float* __restrict__ part, int64_t D, const Chunks ch,
                                                            int together, float* __restrict__ dscale,
                                                            float* __restrict__ dshift) {
  typedef float vec __attribute__((ext_vector_type(V)));
  __shared__ vec red[16][17];
  const int col = threadIdx.x % 16, strand = threadIdx.x / 16;
  const int64_t i = (int64_t(blockIdx.x) * 16 + col) * V;
  float* out = blockIdx.z ? dshift : dscale;
  if (!out) return;
  int c0 = 0, c1 = ch.first[kMaxSeqs];
  if (!together) {
#pragma unroll
    for (int b = 0; b < kMaxSeqs; ++b)
      if (b == int(blockIdx.y)) {
        c0 = ch.first[b];
        c1 = ch.first[b + 1];
      }
  }
  vec v = 0.f;
  if (i < D) {
    const float* p = part + blockIdx.z * D + i;
    int c = c0 + strand;
    for (; c + 64 * 3 < c1; c += 64 * 4) {   // four loads in flight
      vec t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = *reinterpret_cast<const vec*>(p + 2 * D * (c + 64 * k));
#pragma unroll
      for (int k = 0; k < 4; ++k) v += t[k];
    }
    for (; c < c1; c += 64) v += *reinterpret_cast<const vec*>(p + 2 * D * c);
  }
  // A wave's four strands, then the sixteen waves.
#pragma unroll
  for (int k = 16; k < kWave; k *= 2)
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += __shfl_xor(v[e], k);
  if (strand % 4 == 0) red[strand / 4][col] = v;
  __syncthreads();
  if (strand == 0 && i < D) {
#pragma unroll
    for (int k = 1; k < 16; ++k) v += red[k][col];
    float* o = out + int64_t(blockIdx.y) * D + i;
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = v[e];
  }
}

int check_norm(const char* who, int64_t M, int64_t D, int32_t B, const int64_t* off, int64_t mod_stride, int dtype,
               Images& im) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 25), "%s: M=%lld outside [0, 2^25)", who, (long long)M);
  AVITS_REQUIRE(D >= 1 && D <= 65536, "%s: D=%lld outside [1, 65536]", who, (long long)D);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  return fill_images(who, M, B, off, mod_stride, im);
}

// Chunks of rows at most, of at least four rows: whole rounds of workgroups with two
// waves to a SIMD or a little more, by the waves that rows of bf16 take.  Measured, 512
// chunks and by this rule: 40000 x 512 bf16 51.8 and 38.3 us, 16000 x 37 24.3
// and 15.5, 4608 x 4096 34.8 and 30.3.  Rows held in 8 bits that take eight waves run in
// twice as many, one row at a time, so that two workgroups fit a CU: 16000 x 4096 76.4
// us instead of 89.3 (rows as they were: 89.1 instead of 86.2).
int64_t max_chunks(int64_t D, bool held) {
  return 256 * ceil_div64(8, std::min<int64_t>(held && D <= 4096 ? 7 : 8, ceil_div64(D, 512)));
}

Chunks make_chunks(int64_t M, int64_t D, bool held, const Images& im) {
  Chunks ch;
  ch.rows = int32_t(std::max<int64_t>(4, ceil_div64(M, max_chunks(D, held))));
  int64_t longest = 0;
  for (int i = 0; i < im.B; ++i) longest = std::max(longest, im.end[i] - (i ? im.end[i - 1] : 0));
  // Few rows go as one chunk, whose sums need no second launch: a call with 8 x 2048 bf16
  // 8.4 us instead of 11.5 (with 16 rows 11.5 either way, with 32 20.9 instead of 11.7).
  if (longest <= 8) ch.rows = 8;
  int32_t n = 0;
  int64_t at = 0;
  for (int i = 0; i < kMaxSeqs; ++i) {
    ch.first[i] = n;
    if (i < im.B) n += int32_t(std::max<int64_t>(1, ceil_div64(im.end[i] - at, ch.rows)));
    at = im.end[i];
  }
  ch.first[kMaxSeqs] = n;
  return ch;
}

template <typename T>
void run_norm(const void* x, int64_t M, int64_t D, const Images& im, const void* shift, const void* scale, float eps,
              void* h, float* mean, float* rstd, hipStream_t s) {
  TimedLaunch timed("layer_norm", s);
  const T *px = static_cast<const T*>(x), *sh = static_cast<const T*>(shift), *sc = static_cast<const T*>(scale);
  T* ph = static_cast<T*>(h);
  const int64_t chunks = ceil_div64(D * int64_t(sizeof(T)), 16 * kWave);   // a wave's chunks per lane
  if (D < kVec<T> || chunks > 32) {
    hipLaunchKernelGGL(norm_any_kernel<T>, dim3(unsigned(ceil_div64(M, 4))), dim3(256), 0, s, px, M, D, im, sh, sc, eps, ph,
                       mean, rstd);
    return;
  }
  auto go = [&](auto nc, auto waves) {
    constexpr int kNC = decltype(nc)::value, kW = decltype(waves)::value;
    const int64_t teams = 4 / kW;
    // A few rows to a team, once there are enough for every SIMD.
    const int per = int(std::min<int64_t>(8, std::max<int64_t>(1, M / (teams * 2048))));
    const dim3 grid(unsigned(ceil_div64(M, teams * per)));
    if (D % kVec<T> == 0)
      hipLaunchKernelGGL((norm_rows_kernel<T, kNC, kW, false>), grid, dim3(256), 0, s, px, M, D, im, sh, sc, eps, ph, mean, rstd,
                         per);
    else
      hipLaunchKernelGGL((norm_rows_kernel<T, kNC, kW, true>), grid, dim3(256), 0, s, px, M, D, im, sh, sc, eps, ph, mean, rstd,
                         per);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 4> four;
  // One wave to a row while a lane holds four chunks at most, else four: 16000 x
  // 2050 bf16 38.9 us, by one wave 59.1; one such row 3.8 and 7.3.
  if (chunks <= 1) go(one, one);
  else if (chunks <= 2) go(integral_constant<int, 2>(), one);
  else if (chunks <= 4) go(four, one);
  else if (chunks <= 8) go(integral_constant<int, 2>(), four);
  else if (chunks <= 16) go(four, four);
  else go(integral_constant<int, 8>(), four);
}

template <typename T>
void run_norm_back(const void* dh, const Rows<T>& rows, const float* mean, const float* rstd, int64_t M, int64_t D,
                   const Images& im, const void* scale, const void* dres, void* dx, float* dscale, float* dshift,
                   float* ws, hipStream_t s) {
  TimedLaunch timed("layer_norm_backward", s);
  const Chunks ch = make_chunks(M, D, rows.q != nullptr, im);
  const int n = ch.first[kMaxSeqs];
  float* avg = ws;
  float* part = ws + align_up(size_t(2 * M), 64);
  const T *d = static_cast<const T*>(dh), *sc = static_cast<const T*>(scale), *res = static_cast<const T*>(dres);
  T* o = static_cast<T*>(dx);
  // One chunk for each gradient's vector: its sums are the gradient.
  const bool direct = n == (im.stride == 0 ? 1 : im.B), wanted = dscale || dshift;
  const SumsOut sums = direct || !wanted ? SumsOut{dscale, dshift, D} : SumsOut{part, part + D, 2 * D};
  const int64_t chunks = ceil_div64(D * int64_t(sizeof(T)), 16);
  if (D >= kVec<T> && chunks <= 2048) {
    auto go = [&](auto nc, auto two) {
      constexpr int kNC = decltype(nc)::value, kR = decltype(two)::value ? 2 : 1;
      const dim3 wg(unsigned(ceil_div64(ceil_div64(chunks, kNC), kWave) * kWave));
      auto form = [&](auto held, auto tail) {
        hipLaunchKernelGGL((norm_back_rows_kernel<T, decltype(held)::value, kNC, kR, decltype(tail)::value>), dim3(unsigned(n)), wg,
                           0, s, d, rows, mean, rstd, D, im, ch, sc, res, o, sums);
      };
      const std::true_type yes;
      const std::false_type no;
      if (rows.q && D % kVec<T> == 0) form(yes, no);
      else if (rows.q) form(yes, yes);
      else if (D % kVec<T> == 0) form(no, no);
      else form(no, yes);
    };
    // Two rows at a time; one where a second workgroup would not fit the CU with two
    // rows' registers: five to seven waves (16000 x 2560 bf16 in 8 bits 53.9 us instead
    // of 79.7), and eight where there are two of them (see max_chunks; with one, 16000 x
    // 3999 rows as they were take 100.9 one at a time, 90.8 by twos).
    const std::integral_constant<int, 1> one;
    if (chunks <= 256 || (chunks > 448 && chunks <= 512 && !rows.q)) go(one, std::true_type());
    else if (chunks <= 512) go(one, std::false_type());
    else if (chunks <= 1024) go(std::integral_constant<int, 2>(), std::false_type());
    else go(std::integral_constant<int, 4>(), std::false_type());
  } else {
    if (M > 0)
      hipLaunchKernelGGL(norm_back_avg_kernel<T>, dim3(unsigned(ceil_div64(M, 4))), dim3(256), 0, s, d, rows, mean, rstd, M, D,
                         im, sc, avg);
    hipLaunchKernelGGL(norm_back_any_kernel<T>, dim3(unsigned(n), unsigned(ceil_div64(D, 256))), dim3(256), 0, s, d, rows,
                       mean, rstd, D, im, ch, sc, res, (const float*)avg, o, sums);
  }
  if (wanted && !direct) {
    const int together = im.stride == 0 ? 1 : 0;
    auto sum = [&](auto v) {
      constexpr int kV = decltype(v)::value;
      hipLaunchKernelGGL(norm_back_sum_kernel<kV>, dim3(unsigned(ceil_div64(D, 16 * kV)), unsigned(together ? 1 : im.B), 2),
                         dim3(1024), 0, s, (const float*)part, D, ch, together, dscale, dshift);
    };
    if (D % 4 == 0 && aligned_to({part}, 16)) sum(std::integral_constant<int, 4>());
    else sum(std::integral_constant<int, 1>());
  }
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" int avits_layer_norm(const void* x, int64_t M, int64_t D, int32_t B, const int64_t* off, const void* shift,
                                const void* scale, int64_t mod_stride, float eps, int dtype, void* h, float* mean,
                                float* rstd, void* stream) {
  Images im;
  const int rc = check_norm("layer_norm", M, D, B, off, mod_stride, dtype, im);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(std::isfinite(eps) && eps > 0.f, "layer_norm: eps=%g must be positive and finite", eps);
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(x && h, "layer_norm: null x/h");
  const size_t z = dtype == AVITS_BF16 ? 2 : 4;
  AVITS_REQUIRE(aligned_to({x, h, shift, scale}, z) && aligned_to({mean, rstd}, 4),
                "layer_norm: a pointer is not aligned to its element");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == AVITS_BF16) run_norm<bf16_t>(x, M, D, im, shift, scale, eps, h, mean, rstd, s);
  else run_norm<float>(x, M, D, im, shift, scale, eps, h, mean, rstd, s);
  return launch_status("layer_norm");
}

extern "C" size_t avits_layer_norm_backward_workspace_bytes(int64_t M, int64_t D, int32_t B) {
  if (M < 0 || M >= (int64_t(1) << 25) || D < 1 || D > 65536 || B < 1 || B > kMaxSeqs) return 0;
  const size_t chunks = size_t(std::min<int64_t>(max_chunks(D, true), ceil_div64(M, 4))) + size_t(B);
  return (align_up(size_t(2 * M), 64) + 2 * chunks * size_t(D)) * sizeof(float);
}

extern "C" int avits_layer_norm_backward(const void* dh, const void* x, const uint8_t* x_q8, const uint8_t* x_s8,
                                         const float* mean, const float* rstd, int64_t M, int64_t D, int32_t B,
                                         const int64_t* off, const void* scale, int64_t mod_stride, const void* dres,
                                         int dtype, void* dx, float* dscale, float* dshift, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  Images im;
  const int rc = check_norm("layer_norm_backward", M, D, B, off, mod_stride, dtype, im);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(M == 0 || ((x != nullptr) != (x_q8 != nullptr) && (x_q8 != nullptr) == (x_s8 != nullptr)),
                "layer_norm_backward: give either x or both x_q8 and x_s8");
  AVITS_REQUIRE(M == 0 || (dh && mean && rstd && dx), "layer_norm_backward: null dh/mean/rstd/dx");
  if (M == 0 && !dscale && !dshift) return AVITS_OK;
  const size_t z = dtype == AVITS_BF16 ? 2 : 4;
  AVITS_REQUIRE(aligned_to({dh, x, scale, dres, dx}, z) && aligned_to({mean, rstd, dscale, dshift, workspace}, 4),
                "layer_norm_backward: a pointer is not aligned to its element");
  const size_t need = avits_layer_norm_backward_workspace_bytes(M, D, B);
  if (!workspace || workspace_bytes < need)
    return set_error(AVITS_ERR_WORKSPACE, "layer_norm_backward: workspace of %zu bytes, need %zu", workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* ws = static_cast<float*>(workspace);
  const int64_t ns = ceil_div64(D, kBlk);
  if (dtype == AVITS_BF16)
    run_norm_back<bf16_t>(dh, {static_cast<const bf16_t*>(x), x_q8, x_s8, ns}, mean, rstd, M, D, im, scale, dres, dx, dscale,
                          dshift, ws, s);
  else
    run_norm_back<float>(dh, {static_cast<const float*>(x), x_q8, x_s8, ns}, mean, rstd, M, D, im, scale, dres, dx, dscale,
                         dshift, ws, s);
  return launch_status("layer_norm_backward");
}
