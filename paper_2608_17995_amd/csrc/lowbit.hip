// Conversions to and from the block-scaled formats, and the GELU's gradient
// from an activation kept in 8 bits.  Every kernel here moves its data once;
// what bounds them is HBM bandwidth, and the launch for a few rows.
#include <type_traits>

#include "kernels.h"
#include "lowbit.h"

namespace avits {
namespace {

// ----------------------------------------------------------------------------
// 8-bit activations: codes [M, D], scales [M, ceil(D / 32)].

// D a multiple of 32, 16-byte aligned: blocks lie one after another through the
// whole array.  A lane takes eight elements, four lanes a block.  4608 x 8192 of
// bf16: 21.8 us for 115 MB (5.3 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void pack8_kernel(const T* __restrict__ x, int64_t n8, uint8_t* __restrict__ q,
                                                    uint8_t* __restrict__ s) {
  // n8 is a multiple of 4: a block's lanes stay together.
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n8; i += int64_t(gridDim.x) * 256) {
    float v[8];
    load8(x + 8 * i, v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[e]));
    top = quad_umax(top);
    const uint32_t c = scale8_code(top);
    const float inv = c == 255u ? 0.f : scale_inverse(c);
    reinterpret_cast<u32x2*>(q)[i] = u32x2{encode8x4(v, inv), encode8x4(v + 4, inv)};
    if (i % 4 == 0) s[i / 4] = uint8_t(c);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack8_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                      int64_t n8, T* __restrict__ x) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n8; i += int64_t(gridDim.x) * 256) {
    const u32x2 c = reinterpret_cast<const u32x2*>(q)[i];
    const float sc = scale_value(s[i / 4]);
    float v[8];
    decode8x4(c[0], sc, v);
    decode8x4(c[1], sc, v + 4);
    store8(x + 8 * i, v);
  }
}

// Any width and alignment: 2^lg lanes walk a row, eight elements each at a time, so
// that four lanes hold a block here too.  The eight of a row's last, partial
// group are the row's last eight: the first `dup` of them belong to the group before
// it, whose lane gives them the same values, where both are of one block; where
// they are not (or the row is shorter) the group goes element by element.
// Bound by HBM like the whole blocks' kernels: 16000 x 3999 of bf16 packed in 43.7 us
// (its bytes at the copy's rate 37.6), their GELU gradient 74.9 (62.7); a lane
// per element took 185 and 216.
struct RowGroup {
  int64_t at;      // where the eight elements start
  int own, dup;    // how many are the group's own (0: past the row), and the first of them
  bool single;     // element by element
};
__device__ __forceinline__ RowGroup row_group(int64_t row, int g, int D) {
  RowGroup r;
  r.own = max(0, min(8, D - 8 * g));
  r.single = r.own < 8 && (g % 4 == 0 || D < 8);
  r.dup = D < 8 ? 0 : 8 - r.own;
  r.at = row * D + 8 * g - r.dup;
  return r;
}
template <typename T>
__device__ __forceinline__ void load_group(const T* x, const RowGroup& r, int D, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (D >= 8) {
    if (r.own > 0) load8(x + r.at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < r.own) v[e] = ld(x, r.at + e);
  }
}
template <typename T>
__device__ __forceinline__ void store_group(T* x, const RowGroup& r, const float (&v)[8]) {
  if (!r.single) {
    if (r.own > 0) store8(x + r.at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= r.dup && e - r.dup < r.own) st(x, r.at + e, v[e]);
  }
}
// The group's values from its codes and its block's scale (a single group's
// first `dup` are of another block and not used).
__device__ __forceinline__ void decode_group(const uint8_t* q, const RowGroup& r, int D, uint32_t c, float (&v)[8]) {
  loose2 w = {0u, 0u};
  if (D >= 8) {
    if (r.own > 0) w = *reinterpret_cast<const loose2*>(q + r.at);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < r.own) w[e / 4] |= uint32_t(q[r.at + e]) << (8 * (e % 4));
  }
  const float sc = scale_value(c);
  decode8x4(w[0], sc, v);
  decode8x4(w[1], sc, v + 4);
}
// f(row, g, group) for the row groups of this thread; where rows are few, gridDim.y
// walks share one.
template <typename F>
__device__ __forceinline__ void each_group(int64_t M, int D, int ns, int lg, F f) {
  const int lanes = 1 << lg, from = int(blockIdx.y) * lanes + (threadIdx.x & (lanes - 1)), step = int(gridDim.y) * lanes;
  for (int64_t row = (int64_t(blockIdx.x) * 256 + threadIdx.x) >> lg; row < M; row += int64_t(gridDim.x) * 256 >> lg)
    for (int g = from; g < 4 * ns; g += step) f(row, g, row_group(row, g, D));
}

template <typename T>
__global__ __launch_bounds__(256) void pack8_rows_kernel(const T* __restrict__ x, int64_t M, int D, int ns, int lg,
                                                         uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  each_group(M, D, ns, lg, [&](int64_t row, int g, const RowGroup& r) {
    float v[8];
    load_group(x, r, D, v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, e >= r.dup ? magnitude(v[e]) : 0u);
    const uint32_t c = scale8_code(quad_umax(top));
    const float inv = c == 255u ? 0.f : scale_inverse(c);
    const loose2 o = {encode8x4(v, inv), encode8x4(v + 4, inv)};
    if (!r.single) {
      if (r.own > 0) *reinterpret_cast<loose2*>(q + r.at) = o;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= r.dup && e - r.dup < r.own) q[r.at + e] = uint8_t(o[e / 4] >> (8 * (e % 4)));
    }
    if (g % 4 == 0) s[row * ns + g / 4] = uint8_t(c);
  });
}

template <typename T>
__global__ __launch_bounds__(256) void unpack8_rows_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                           int64_t M, int D, int ns, int lg, T* __restrict__ x) {
  each_group(M, D, ns, lg, [&](int64_t row, int g, const RowGroup& r) {
    float v[8];
    decode_group(q, r, D, s[row * ns + g / 4], v);
    store_group(x, r, v);
  });
}

// dm = da gelu'(m), m in its own type or kept in 8 bits.  4608 x 8192 of bf16 from
// 8 bits: 32.5 us for 190 MB (5.9 TB/s, partly from the caches).
template <typename T, bool HELD>
__global__ __launch_bounds__(256) void gelu_back_kernel(const T* da, const T* m, const uint8_t* __restrict__ q,
                                                        const uint8_t* __restrict__ s, int64_t n8, T* dm) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n8; i += int64_t(gridDim.x) * 256) {
    float d[8], v[8];
    load8(da + 8 * i, d);
    if constexpr (HELD) {
      const u32x2 c = reinterpret_cast<const u32x2*>(q)[i];
      const float sc = scale_value(s[i / 4]);
      decode8x4(c[0], sc, v);
      decode8x4(c[1], sc, v + 4);
    } else {
      load8(m + 8 * i, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] *= gelu_slope(v[e]);
    store8(dm + 8 * i, d);
  }
}

// (dm may be da: a group's eight and the group's before it are of one block, so
// they are loaded by one instruction before either's are stored.)
template <typename T>
__global__ __launch_bounds__(256) void gelu_back_rows_kernel(const T* da, const T* m, const uint8_t* __restrict__ q,
                                                             const uint8_t* __restrict__ s, int64_t M, int D, int ns, int lg,
                                                             T* dm) {
  each_group(M, D, ns, lg, [&](int64_t row, int g, const RowGroup& r) {
    float d[8], v[8];
    load_group(da, r, D, d);
    if (m) load_group(m, r, D, v);
    else decode_group(q, r, D, s[row * ns + g / 4], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] *= gelu_slope(v[e]);
    store_group(dm, r, d);
  });
}

// ----------------------------------------------------------------------------
// Microscaled 4-bit floats: codes [M, K / 2], scales [ceil(K / 64), Mp, 2] with
// Mp = M rounded up to 8: the two scales of 64 columns of a row side by side,
// the rows one after another, so that a lane of the product that owns several
// consecutive rows reads their scales at once.
//
// A workgroup converts kQRows x kQCols elements: a wave 512 columns of a row at a
// time (a lane eight elements, four lanes a block), the scales turned round
// through LDS so that each pair's rows leave in one run.  16384 x 4096 of bf16: 43.7 us
// for 170 MB (3.9 TB/s), back 28.4 (6.0, partly from the caches).  (32 rows x
// 512 columns to a workgroup: there and back 78 us instead of 72.)
constexpr int kQRows = 16, kQCols = 1024, kQSegs = kQCols / 512, kQItems = kQRows * kQSegs / 4;
static_assert(kQRows * (kQCols / 64) == 256, "one scale pair per thread");

template <typename T, bool GELU>
__global__ __launch_bounds__(256) void quantize4_kernel(const T* __restrict__ x, int64_t M, int64_t K,
                                                        uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  __shared__ uint16_t sc[kQCols / 64][kQRows];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t m0 = int64_t(blockIdx.x) * kQRows, k0 = int64_t(blockIdx.y) * kQCols + 8 * lane;
  const int64_t Mp = scale_rows(M);
#pragma unroll
  for (int r = 0; r < kQItems; ++r) {
    const int row = (wave * kQItems + r) / kQSegs, seg = r % kQSegs;
    const int64_t m = m0 + row, k = k0 + 512 * seg;
    const bool in = k < K && m < M;  // K is a multiple of 32: all four lanes of a block, or none
    float v[8] = {};
    if (in) load8(x + m * K + k, v);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (GELU) v[e] = gelu_value(v[e]);
      top = max(top, magnitude(v[e]));
    }
    const uint32_t c = scale4_code(quad_umax(top));
    const uint32_t o = encode4x8(v, c == 255u ? 0.f : scale_inverse(c));
    if (in) *reinterpret_cast<uint32_t*>(q + (m * K + k) / 2) = o;
    // Lane 8 j: its own block's scale and, from lane 8 j + 7, the next block's.
    const uint32_t up = uint32_t(__builtin_amdgcn_update_dpp(0, int(c), kDppHalfMirror, 0xf, 0xf, false));
    if (lane % 8 == 0) sc[seg * 8 + lane / 8][row] = uint16_t(c | up << 8);
  }
  __syncthreads();
  const int pair = threadIdx.x / kQRows, row = threadIdx.x % kQRows;
  const int64_t gp = int64_t(blockIdx.y) * (kQCols / 64) + pair, m = m0 + row;
  if (gp < scale_groups(K) && m < Mp) reinterpret_cast<uint16_t*>(s)[gp * Mp + m] = sc[pair][row];
}

template <typename T>
__global__ __launch_bounds__(256) void dequantize4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                          int64_t M, int64_t K, T* __restrict__ x) {
  __shared__ uint16_t sc[kQCols / 64][kQRows];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t m0 = int64_t(blockIdx.x) * kQRows, k0 = int64_t(blockIdx.y) * kQCols + 8 * lane;
  const int64_t Mp = scale_rows(M);
  {
    const int pair = threadIdx.x / kQRows, row = threadIdx.x % kQRows;
    const int64_t gp = int64_t(blockIdx.y) * (kQCols / 64) + pair, m = m0 + row;
    sc[pair][row] = gp < scale_groups(K) && m < Mp ? reinterpret_cast<const uint16_t*>(s)[gp * Mp + m] : uint16_t(0);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kQItems; ++r) {
    const int row = (wave * kQItems + r) / kQSegs, seg = r % kQSegs;
    const int64_t m = m0 + row, k = k0 + 512 * seg;
    if (m >= M || k >= K) continue;
    float v[8];
    const uint32_t c = sc[seg * 8 + lane / 8][row] >> (lane & 4 ? 8 : 0);
    decode4x8(*reinterpret_cast<const uint32_t*>(q + (m * K + k) / 2), scale_value(c & 255u), v);
    store8(x + m * K + k, v);
  }
}

int check_type(const char* who, int64_t M, int64_t D, int dtype) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 31), "%s: M=%lld outside [0, 2^31)", who, (long long)M);
  AVITS_REQUIRE(D >= 1 && D < (int64_t(1) << 24), "%s: D=%lld outside [1, 2^24)", who, (long long)D);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  return AVITS_OK;
}

bool vectors_ok(int64_t D, std::initializer_list<const void*> wide, const void* codes) {
  return D % kBlk == 0 && aligned_to(wide, 16) && aligned_to({codes}, 8);
}

constexpr int64_t kMaxGrid = 1 << 22;  // workgroups; beyond it the kernels loop
// Lanes that walk a row of 4 ns groups: as many of a wave as keep four fifths of
// them busy.
int row_lanes_log2(int64_t ns) {
  int lg = 6;
  while (lg > 2 && (ceil_div64(4 * ns, int64_t(1) << lg) << lg) * 4 > 4 * ns * 5) --lg;
  return lg;
}
// A thread to each group while there are fewer than 2^19 (1741 x 3999 bf16 values
// packed: 6.6 us, with one walk to a row 9.1; 300 x 3999: 3.3 and 6.4).
dim3 rows_grid(int64_t M, int64_t ns, int lg) {
  const int64_t walks = std::min(ceil_div64(4 * ns, int64_t(1) << lg), std::max<int64_t>(1, (int64_t(1) << 19) / (M << lg)));
  return dim3(unsigned(std::min(kMaxGrid, ceil_div64(M << lg, 256))), unsigned(walks));
}
dim3 flat_grid(int64_t n8) { return dim3(unsigned(std::min(kMaxGrid, ceil_div64(n8, 256)))); }

template <typename F>
int by_type(int dtype, F f) {
  if (dtype == AVITS_BF16) f(bf16_t{});
  else f(float{});
  return AVITS_OK;
}

int check_mx(const char* who, int64_t M, int64_t K, int dtype) {
  const int rc = check_type(who, M, K, dtype);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(M < (int64_t(1) << 27), "%s: M=%lld is 2^27 or more", who, (long long)M);
  AVITS_REQUIRE(K % kBlk == 0, "%s: K=%lld must be a multiple of 32", who, (long long)K);
  AVITS_REQUIRE(scale_groups(K) * scale_rows(M) * 2 < (int64_t(1) << 31), "%s: M=%lld x K=%lld has 2^31 scales or more", who,
                (long long)M, (long long)K);
  return AVITS_OK;
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" int avits_ckpt8_pack(const void* x, int64_t M, int64_t D, int dtype, uint8_t* q, uint8_t* s, void* stream) {
  const int rc = check_type("ckpt8_pack", M, D, dtype);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(x && q && s, "ckpt8_pack: null x/q/s");
  AVITS_REQUIRE(aligned_to({x}, dtype == AVITS_BF16 ? 2 : 4), "ckpt8_pack: x is not aligned to its element");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int ns = int(ceil_div64(D, kBlk)), lg = row_lanes_log2(ns);
  TimedLaunch timed("ckpt8", st);
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const T* p = static_cast<const T*>(x);
    if (vectors_ok(D, {x}, q))
      hipLaunchKernelGGL(pack8_kernel<T>, flat_grid(M * D / 8), dim3(256), 0, st, p, M * D / 8, q, s);
    else
      hipLaunchKernelGGL(pack8_rows_kernel<T>, rows_grid(M, ns, lg), dim3(256), 0, st, p, M, int(D), ns, lg, q, s);
  });
  return launch_status("ckpt8_pack");
}

extern "C" int avits_ckpt8_unpack(const uint8_t* q, const uint8_t* s, int64_t M, int64_t D, int dtype, void* x, void* stream) {
  const int rc = check_type("ckpt8_unpack", M, D, dtype);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(x && q && s, "ckpt8_unpack: null q/s/x");
  AVITS_REQUIRE(aligned_to({x}, dtype == AVITS_BF16 ? 2 : 4), "ckpt8_unpack: x is not aligned to its element");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int ns = int(ceil_div64(D, kBlk)), lg = row_lanes_log2(ns);
  TimedLaunch timed("ckpt8", st);
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    T* p = static_cast<T*>(x);
    if (vectors_ok(D, {x}, q))
      hipLaunchKernelGGL(unpack8_kernel<T>, flat_grid(M * D / 8), dim3(256), 0, st, q, s, M * D / 8, p);
    else
      hipLaunchKernelGGL(unpack8_rows_kernel<T>, rows_grid(M, ns, lg), dim3(256), 0, st, q, s, M, int(D), ns, lg, p);
  });
  return launch_status("ckpt8_unpack");
}

extern "C" int avits_gelu_backward(const void* da, const void* m, const uint8_t* m_q8, const uint8_t* m_s8, int64_t M,
                                   int64_t D, int dtype, void* dm, void* stream) {
  const int rc = check_type("gelu_backward", M, D, dtype);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE((m != nullptr) != (m_q8 != nullptr) && (m_q8 != nullptr) == (m_s8 != nullptr),
                "gelu_backward: give either m or both m_q8 and m_s8");
  AVITS_REQUIRE(da && dm, "gelu_backward: null da/dm");
  AVITS_REQUIRE(aligned_to({da, m, dm}, dtype == AVITS_BF16 ? 2 : 4), "gelu_backward: a pointer is not aligned to its element");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int ns = int(ceil_div64(D, kBlk)), lg = row_lanes_log2(ns);
  TimedLaunch timed("gelu_backward", st);
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const T *d = static_cast<const T*>(da), *v = static_cast<const T*>(m);
    T* o = static_cast<T*>(dm);
    const int64_t n8 = M * D / 8;
    if (!vectors_ok(D, {da, m, dm}, m_q8))
      hipLaunchKernelGGL(gelu_back_rows_kernel<T>, rows_grid(M, ns, lg), dim3(256), 0, st, d, v, m_q8, m_s8, M, int(D), ns, lg, o);
    else if (m_q8)
      hipLaunchKernelGGL((gelu_back_kernel<T, true>), flat_grid(n8), dim3(256), 0, st, d, v, m_q8, m_s8, n8, o);
    else
      hipLaunchKernelGGL((gelu_back_kernel<T, false>), flat_grid(n8), dim3(256), 0, st, d, v, m_q8, m_s8, n8, o);
  });
  return launch_status("gelu_backward");
}

extern "C" size_t avits_mxfp4_scale_bytes(int64_t M, int64_t K) {
  if (M < 0 || M >= (int64_t(1) << 27) || K < kBlk || K >= (int64_t(1) << 24) || K % kBlk != 0) return 0;
  const int64_t bytes = scale_groups(K) * scale_rows(M) * 2;
  return bytes < (int64_t(1) << 31) ? size_t(bytes) : 0;
}

extern "C" int avits_mxfp4_quantize(const void* x, int64_t M, int64_t K, int act, int dtype, uint8_t* q, uint8_t* s,
                                    void* stream) {
  const int rc = check_mx("mxfp4_quantize", M, K, dtype);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(act == AVITS_ACT_NONE || act == AVITS_ACT_GELU, "mxfp4_quantize: act=%d unknown", act);
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(x && q && s, "mxfp4_quantize: null x/q/s");
  AVITS_REQUIRE(aligned_to({x, q, s}, 16), "mxfp4_quantize: x, q and s must be 16-byte aligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid(unsigned(ceil_div64(M, kQRows)), unsigned(ceil_div64(K, kQCols)));
  TimedLaunch timed("mxfp4_quantize", st);
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const T* p = static_cast<const T*>(x);
    if (act == AVITS_ACT_GELU)
      hipLaunchKernelGGL((quantize4_kernel<T, true>), grid, dim3(256), 0, st, p, M, K, q, s);
    else
      hipLaunchKernelGGL((quantize4_kernel<T, false>), grid, dim3(256), 0, st, p, M, K, q, s);
  });
  return launch_status("mxfp4_quantize");
}

extern "C" int avits_mxfp4_dequantize(const uint8_t* q, const uint8_t* s, int64_t M, int64_t K, int dtype, void* x,
                                      void* stream) {
  const int rc = check_mx("mxfp4_dequantize", M, K, dtype);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(x && q && s, "mxfp4_dequantize: null q/s/x");
  AVITS_REQUIRE(aligned_to({x, q, s}, 16), "mxfp4_dequantize: q, s and x must be 16-byte aligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid(unsigned(ceil_div64(M, kQRows)), unsigned(ceil_div64(K, kQCols)));
  TimedLaunch timed("mxfp4_dequantize", st);
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(dequantize4_kernel<T>, grid, dim3(256), 0, st, q, s, M, K, static_cast<T*>(x));
  });
  return launch_status("mxfp4_dequantize");
}
