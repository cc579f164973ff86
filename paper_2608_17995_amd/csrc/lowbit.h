// Device helpers of the block-scaled formats: 32 consecutive elements of a
// row share one power-of-two scale, held as a biased exponent byte c (2^(c -
// 127); 255 stands for NaN).  4-bit elements are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6
// and their negatives), two to a byte, the even one in the low half; 8-bit ones
// are e4m3 (largest 448).
#pragma once

#include <initializer_list>

#include "kernels.h"

namespace avits {
namespace {

// Rows of B images, one image after another, each with its own modulation
// vectors.
struct Images {
  int32_t B;
  int64_t stride;             // elements between the images' vectors
  int64_t end[kMaxSeqs];      // row after each image's last
};

// Image of a row (a loop over kernel arguments: scalar work).
__device__ __forceinline__ int image_of(const Images& im, int64_t row) {
  int b = 0;
#pragma unroll
  for (int i = 0; i < kMaxSeqs - 1; ++i) b += (i < im.B - 1 && row >= im.end[i]) ? 1 : 0;
  return b;
}

inline int fill_images(const char* who, int64_t M, int32_t B, const int64_t* off, int64_t stride, Images& im) {
  AVITS_REQUIRE(B >= 1 && B <= kMaxSeqs, "%s: B=%d outside [1, %d]", who, B, kMaxSeqs);
  AVITS_REQUIRE(off || B == 1, "%s: null off with B=%d", who, B);
  AVITS_REQUIRE(stride >= 0, "%s: mod_stride=%lld < 0", who, (long long)stride);
  im.B = B;
  im.stride = stride;
  for (int i = 0; i < kMaxSeqs; ++i) im.end[i] = M;
  if (!off) return AVITS_OK;
  AVITS_REQUIRE(off[0] == 0 && off[B] == M, "%s: off must run from 0 to M=%lld", who, (long long)M);
  for (int i = 0; i < B; ++i) {
    AVITS_REQUIRE(off[i] <= off[i + 1], "%s: off[%d] > off[%d]", who, i, i + 1);
    im.end[i] = off[i + 1];
  }
  return AVITS_OK;
}

inline bool aligned_to(std::initializer_list<const void*> ps, size_t z) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % z != 0) return false;
  return true;
}

constexpr int kBlk = 32;  // elements that share a scale

__host__ __device__ constexpr int64_t scale_groups(int64_t K) { return (K + 63) / 64; }  // pairs of blocks
__host__ __device__ constexpr int64_t scale_rows(int64_t M) { return (M + 7) / 8 * 8; }

// 2^(c - 127) as fp32 (c = 0 is the subnormal 2^-127).
__device__ __forceinline__ float scale_value(uint32_t c) {
  return __uint_as_float(c == 255u ? 0x7fc00000u : c == 0u ? 0x00400000u : c << 23);
}
// 2^(127 - c), c <= 253: what elements are multiplied with before they are rounded.
__device__ __forceinline__ float scale_inverse(uint32_t c) { return __uint_as_float((254u - c) << 23); }

// The scale byte of a block whose largest magnitude has the bit pattern `top`.
// 4-bit: 2^(floor(log2 top) - 2), the exponent of 6 on the block's largest
// (values between 6 and 8 scales become 6, the format's usual rule).  8-bit: the smallest
// power of two that leaves the largest at most 448, so that no element is cut
// off and every rounding is within half a step.  A block that holds an infinity
// or a NaN gets 255: all of it reads back as NaN.
__device__ __forceinline__ uint32_t scale4_code(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : e < 2u ? 0u : e - 2u;
}
__device__ __forceinline__ uint32_t scale8_code(uint32_t top) {
  const uint32_t e = top >> 23, c = e + ((top & 0x7fffffu) > 0x600000u ? 1u : 0u);
  return e == 255u ? 255u : c < 8u ? 0u : c - 8u;
}

// Largest of a value over aligned groups of 4 lanes, every lane receiving it.
__device__ __forceinline__ uint32_t quad_umax(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), kDppXor1, 0xf, 0xf, false)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), kDppXor2, 0xf, 0xf, false)));
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Vectors of memory that need not start on their own size: global accesses of
// 16 bytes may lie at any element (or byte).
typedef uint32_t loose4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t loose2 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t loose1 __attribute__((aligned(1)));

// Eight elements to eight 4-bit codes (round to nearest even, magnitudes past 6 to 6).
__device__ __forceinline__ uint32_t encode4x8(const float (&v)[8], float inv) {
  uint32_t o = 0;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[0] * inv, v[1] * inv, 1.f, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[2] * inv, v[3] * inv, 1.f, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[4] * inv, v[5] * inv, 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[6] * inv, v[7] * inv, 1.f, 3);
}
__device__ __forceinline__ void decode4x8(uint32_t c, float scale, float (&v)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3);
  v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
  v[4] = d[0] * scale; v[5] = d[1] * scale; v[6] = e[0] * scale; v[7] = e[1] * scale;
}

// Four elements to e4m3 codes (round to nearest even) and back.
__device__ __forceinline__ uint32_t encode8x4(const float* v, float inv) {
  int o = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, o, true));
}
__device__ __forceinline__ void decode8x4(uint32_t c, float scale, float* v) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), true);
  v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
}
__device__ __forceinline__ float decode8(uint8_t c, float scale) {
  return __builtin_amdgcn_cvt_f32_fp8(int(c), 0) * scale;
}

// Eight consecutive elements as floats, and back (no alignment but the element's).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const loose4 w = *reinterpret_cast<const loose4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
    const loose4 a = *reinterpret_cast<const loose4*>(p), b = *reinterpret_cast<const loose4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = __uint_as_float(a[e]);
      v[4 + e] = __uint_as_float(b[e]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<loose4*>(p) =
        loose4{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7])};
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<loose4*>(p + 4 * h) = loose4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]),
                                                     __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
  }
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// GELU with the tanh approximation, x s(2u) with the logistic function s and
// u = sqrt(2 / pi) (x + 0.044715 x^3), and its derivative
// s + x s (1 - s) 2 u'.  exp2 and the reciprocal are the hardware's (about 1 ulp).
__device__ __forceinline__ float gelu_exp(float x) {  // exp(-2u)
  return __builtin_amdgcn_exp2f(-2.302208198f * x * fmaf(0.044715f * x, x, 1.f));
}
__device__ __forceinline__ float gelu_value(float x) {
  const float s = __builtin_amdgcn_rcpf(1.f + gelu_exp(x));
  return s == 0.f ? -0.f : x * s;  // also at minus infinity
}
__device__ __forceinline__ float gelu_slope(float x) {
  const float e = gelu_exp(x), s = __builtin_amdgcn_rcpf(1.f + e);
  // s (1 - s) as s (s e): 1 - s keeps no digits where s is near 1.  Where it is
  // 0 so is the second term, also where x 2u' overflows.
  const float t = s == 0.f ? 0.f : s * (s * e);
  return t == 0.f ? s : fmaf(x * (1.5957691216f * fmaf(0.134145f * x, x, 1.f)), t, s);
}

}  // namespace
}  // namespace avits
