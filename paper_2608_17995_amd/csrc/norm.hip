// The modulated layer norm with its statistics, and its backward pass.
//
//   n = (x - mean) rstd,   h = n (1 + scale) + shift
//   g = dh (1 + scale),    dx = rstd (g - avg(g) - n avg(g n)) [+ dres]
//   dscale = sum over rows of dh n,   dshift = sum over rows of dh
//
// Rows of several images lie one after another; image b's rows take the
// vectors b * mod_stride elements after the first image's.
#include <cmath>

#include "kernels.h"
#include "lowbit.h"

namespace avits {
namespace {

template <typename T>
__device__ __forceinline__ float one_or(const T* p, int64_t i) { return p ? 1.f + ld(p, i) : 1.f; }

// Any width and alignment: a wave per row, elements one by one, the row read
// three times (it stays in the caches).
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

// Backward, any width and alignment, in two steps: the two averages of each row
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
                                                            const float* __restrict__ avg, T* dx, float* __restrict__ part,
                                                            int parts) {
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
  if (parts) {
    part[int64_t(2 * c) * D + i] = sc;
    part[int64_t(2 * c + 1) * D + i] = sh;
  }
}

// Sums of the chunks' parts, in chunk order within each of 16 strands: 16
// columns of a workgroup, blockIdx.y the image (or all of them together),
// blockIdx.z scale or shift.
__global__ __launch_bounds__(256) void norm_back_sum_kernel(const float* __restrict__ part, int64_t D, const Chunks ch,
                                                            int together, float* __restrict__ dscale,
                                                            float* __restrict__ dshift) {
  __shared__ float red[16][17];
  const int col = threadIdx.x % 16, strand = threadIdx.x / 16;
  const int64_t i = int64_t(blockIdx.x) * 16 + col;
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
  float v = 0.f;
  if (i < D)
    for (int c = c0 + strand; c < c1; c += 16) v += part[int64_t(2 * c + blockIdx.z) * D + i];
  red[strand][col] = v;
  __syncthreads();
  if (strand == 0 && i < D) {
#pragma unroll
    for (int k = 1; k < 16; ++k) v += red[k][col];
    out[int64_t(blockIdx.y) * D + i] = v;
  }
}

int check_norm(const char* who, int64_t M, int64_t D, int32_t B, const int64_t* off, int64_t mod_stride, int dtype,
               Images& im) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 26), "%s: M=%lld outside [0, 2^26)", who, (long long)M);
  AVITS_REQUIRE(D >= 1 && D <= 65536, "%s: D=%lld outside [1, 65536]", who, (long long)D);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  return fill_images(who, M, B, off, mod_stride, im);
}

constexpr int kMaxChunks = 512;  // two workgroups per CU

Chunks make_chunks(int64_t M, const Images& im) {
  Chunks ch;
  ch.rows = int32_t(std::max<int64_t>(4, ceil_div64(M, kMaxChunks)));
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
  hipLaunchKernelGGL(norm_any_kernel<T>, dim3(unsigned(ceil_div64(M, 4))), dim3(256), 0, s, static_cast<const T*>(x), M, D,
                     im, static_cast<const T*>(shift), static_cast<const T*>(scale), eps, static_cast<T*>(h), mean, rstd);
}

template <typename T>
void run_norm_back(const void* dh, const Rows<T>& rows, const float* mean, const float* rstd, int64_t M, int64_t D,
                   const Images& im, const void* scale, const void* dres, void* dx, float* dscale, float* dshift,
                   float* ws, hipStream_t s) {
  TimedLaunch timed("layer_norm_backward", s);
  const Chunks ch = make_chunks(M, im);
  const int n = ch.first[kMaxSeqs];
  float* avg = ws;
  float* part = ws + align_up(size_t(2 * M), 64);
  const T *d = static_cast<const T*>(dh), *sc = static_cast<const T*>(scale);
  if (M > 0)
    hipLaunchKernelGGL(norm_back_avg_kernel<T>, dim3(unsigned(ceil_div64(M, 4))), dim3(256), 0, s, d, rows, mean, rstd, M, D,
                       im, sc, avg);
  hipLaunchKernelGGL(norm_back_any_kernel<T>, dim3(unsigned(n), unsigned(ceil_div64(D, 256))), dim3(256), 0, s, d, rows, mean,
                     rstd, D, im, ch, sc, static_cast<const T*>(dres), (const float*)avg, static_cast<T*>(dx), part,
                     dscale || dshift ? 1 : 0);
  if (dscale || dshift) {
    const int together = im.stride == 0 ? 1 : 0;
    hipLaunchKernelGGL(norm_back_sum_kernel, dim3(unsigned(ceil_div64(D, 16)), unsigned(together ? 1 : im.B), 2), dim3(256), 0,
                       s, (const float*)part, D, ch, together, dscale, dshift);
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
  if (M < 0 || M >= (int64_t(1) << 26) || D < 1 || D > 65536 || B < 1 || B > kMaxSeqs) return 0;
  const size_t chunks = size_t(std::min<int64_t>(kMaxChunks, ceil_div64(M, 4))) + size_t(B);
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
