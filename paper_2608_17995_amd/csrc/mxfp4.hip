// Products with microscaled 4-bit weights.
//
//   out[m, n] = sum_k x[m, k] w[n, k] + b[n], x and w both held in 4 bits
//   dx[m, k]  = sum_n dy[m, n] w[n, k], dy in bf16 or fp32
//
// The scaled matrix instruction takes 128 elements of 16 rows of both operands:
// lane l holds row l % 16, elements 32 (l / 16) .. + 31 (one block) in 16 bytes
// and that block's scale in a byte of a register.  Which 32 elements of the
// contraction a lane group takes is free as long as both operands agree, and so is
// which 16 rows one instruction takes.  Both are used so that operands and scales
// come as they lie in memory: in a step of 256 elements lane group g takes blocks
// 2 g and 2 g + 1 (32 consecutive bytes, and the two scales of one pair), and
// instruction i of a strip of 16 T rows takes rows T l + i, so that a lane's T row
// tiles are T consecutive rows, whose scale pairs are 2 T consecutive bytes.
#include <type_traits>
#include <utility>

#include "kernels.h"
#include "lowbit.h"

namespace avits {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStepK = 256;              // contraction of a step: 128 bytes of a row
constexpr uint32_t kNowhere = 0x80000000u;  // a buffer offset past every range below

__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const void* base, int64_t bytes) {
  const uint32_t n = bytes <= 0 ? 0u : bytes >= int64_t(kNowhere) ? kNowhere : uint32_t(bytes);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, int(n), 0x00020000);
}

// acc += A B^T of 128 elements: byte OA of sa (OB of sb) scales the lane's block.
template <int OA, int OB>
__device__ __forceinline__ f32x4 mfma4(const u32x4& a, const u32x4& b, const f32x4& c, uint32_t sa, uint32_t sb) {
  const i32x8 va = {int(a[0]), int(a[1]), int(a[2]), int(a[3]), 0, 0, 0, 0};
  const i32x8 vb = {int(b[0]), int(b[1]), int(b[2]), int(b[3]), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, OA, int(sa), OB, int(sb));
}

template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  [&]<int... I>(std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
  (std::make_integer_sequence<int, N>());
}

// The scale pairs of T consecutive rows: row i's bytes (block 2 g, 2 g + 1) are
// bytes 2 (i % 2), + 1 of dword i / 2.
template <int T>
struct Pairs {
  uint32_t v[(T + 1) / 2];
};
template <int T>
__device__ __forceinline__ Pairs<T> load_pairs(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  Pairs<T> p;
  if constexpr (T == 1) {
    p.v[0] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r, int(off), 0, 0));
  } else if constexpr (T == 2) {
    p.v[0] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(r, int(off), 0, 0));
  } else if constexpr (T == 4) {
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, int(off), 0, 0));
    p.v[0] = w[0];
    p.v[1] = w[1];
  } else {
    const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, int(off), 0, 0));
    p.v[0] = w[0]; p.v[1] = w[1]; p.v[2] = w[2]; p.v[3] = w[3];
  }
  return p;
}

struct Mx4Args {
  const uint8_t *xq, *xs, *wq, *ws;
  const void *bias, *gate, *resid;
  void* out;
  int64_t M, N, K;
  Images im;  // whose gate a row takes
};

// One output value from its sum: + bias, then optionally resid + gate * (.).
template <typename T>
__device__ __forceinline__ void finish(const Mx4Args& a, int64_t m, int64_t n, float v) {
  if (a.bias) v += ld(static_cast<const T*>(a.bias), n);
  if (a.gate)
    v = ld(static_cast<const T*>(a.resid), m * a.N + n) +
        ld(static_cast<const T*>(a.gate), int64_t(image_of(a.im, m)) * a.im.stride + n) * v;
  st(static_cast<T*>(a.out), m * a.N + n, v);
}

// Few rows: a workgroup of four waves owns 16 TM x 16 TN outputs, the waves
// take every fourth step of the contraction straight from memory into
// registers, and their sums meet in LDS.
template <int TM, int TN, typename T>
__global__ __launch_bounds__(256) void mx4_rows_kernel(const Mx4Args a) {
  __shared__ float red[4][TM * TN * 4][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l = lane % 16, g = lane / 16;
  const int64_t tn = (a.N + 16 * TN - 1) / (16 * TN), tiles = tn * ((a.M + 16 * TM - 1) / (16 * TM));
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t n0 = tile % tn * (16 * TN), m0 = tile / tn * (16 * TM);
    const int64_t Mp = scale_rows(a.M), Np = scale_rows(a.N), groups = scale_groups(a.K);
    const __amdgpu_buffer_rsrc_t rx = range_of(a.xq + m0 * (a.K / 2), (a.M - m0) * (a.K / 2));
    const __amdgpu_buffer_rsrc_t rw = range_of(a.wq + n0 * (a.K / 2), (a.N - n0) * (a.K / 2));
    const __amdgpu_buffer_rsrc_t rxs = range_of(a.xs, groups * Mp * 2), rws = range_of(a.ws, groups * Np * 2);
    const uint32_t rowb = uint32_t(a.K / 2);
    const int steps = int((a.K + kStepK - 1) / kStepK);
    f32x4 acc[TM][TN] = {};
    for (int t = wave; t < steps; t += 4) {
      u32x4 x[TM][2], w[TN][2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t c = uint32_t(t) * 128 + 32 * g + 16 * k;  // byte of the row; past its end nothing is read
#pragma unroll
        for (int j = 0; j < TN; ++j)
          w[j][k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                  rw, int(c < rowb ? (TN * l + j) * rowb + c : kNowhere), 0, 0));
#pragma unroll
        for (int i = 0; i < TM; ++i)
          x[i][k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                  rx, int(c < rowb ? (TM * l + i) * rowb + c : kNowhere), 0, 0));
      }
      const Pairs<TN> sw = load_pairs<TN>(rws, uint32_t(((4 * t + g) * Np + n0 + TN * l) * 2));
      const Pairs<TM> sx = load_pairs<TM>(rxs, uint32_t(((4 * t + g) * Mp + m0 + TM * l) * 2));
      unrolled<2>([&](auto k) {
        unrolled<TM>([&](auto i) {
          unrolled<TN>([&](auto j) {
            acc[i][j] = mfma4<2 * (j % 2) + k, 2 * (i % 2) + k>(w[j][k], x[i][k], acc[i][j], sw.v[j / 2], sx.v[i / 2]);
          });
        });
      });
    }
    // acc[i][j][r] = out[m0 + TM l + i][n0 + TN (4 g + r) + j].
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][(i * TN + j) * 4 + r][lane] = acc[i][j][r];
    __syncthreads();
    // Wave w finishes register w of every accumulator.
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = m0 + TM * l + i;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int at = (i * TN + j) * 4 + wave;
        const float v = (red[0][at][lane] + red[1][at][lane]) + (red[2][at][lane] + red[3][at][lane]);
        const int64_t n = n0 + TN * (4 * g + wave) + j;
        if (m < a.M && n < a.N) finish<T>(a, m, n, v);
      }
    }
    __syncthreads();  // before the next tile's sums
  }
}

// The weight as T values, transposed: wt [K, ld] with zeros in columns N .. ld.
// A workgroup turns 64 rows x 64 columns round in LDS.
template <typename T>
__global__ __launch_bounds__(256) void transpose4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                         int64_t N, int64_t K, T* __restrict__ wt, int64_t ld) {
  __shared__ T tile[64][64 + 16 / sizeof(T)];
  const int64_t n0 = int64_t(blockIdx.x) * 64, k0 = int64_t(blockIdx.y) * 64;
  const int64_t Np = scale_rows(N);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = threadIdx.x / 8 + 32 * h, ch = threadIdx.x % 8;
    const int64_t n = n0 + row, k = k0 + 8 * ch;
    float v[8] = {};
    if (n < N && k < K) {
      const uint8_t c = s[((k / 64) * Np + n) * 2 + (k / 32) % 2];
      decode4x8(*reinterpret_cast<const uint32_t*>(q + (n * K + k) / 2), scale_value(c), v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) st(&tile[0][0], (8 * ch + e) * int64_t(64 + 16 / sizeof(T)) + row, v[e]);
  }
  __syncthreads();
  constexpr int E = 16 / sizeof(T), kLanes = 64 / E;  // 16 bytes per lane
#pragma unroll
  for (int r = threadIdx.x / kLanes; r < 64; r += 256 / kLanes) {
    const int ch = threadIdx.x % kLanes;
    const int64_t k = k0 + r, n = n0 + E * ch;
    if (k < K && n < ld) *reinterpret_cast<u32x4*>(wt + k * ld + n) = *reinterpret_cast<const u32x4*>(&tile[r][E * ch]);
  }
}

// Rows of N elements to rows of ld, zeros behind (any alignment).
template <typename T>
__global__ __launch_bounds__(256) void widen_kernel(const T* __restrict__ x, int64_t M, int64_t N, T* __restrict__ y,
                                                    int64_t ld) {
  const int64_t n = int64_t(blockIdx.y) * 256 + threadIdx.x;
  if (n >= ld) return;
  for (int64_t m = blockIdx.x; m < M; m += gridDim.x) y[m * ld + n] = n < N ? x[m * N + n] : T(0);
}

int check_product(const char* who, int64_t M, int64_t N, int64_t K, int dtype) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 28), "%s: M=%lld outside [0, 2^28)", who, (long long)M);
  AVITS_REQUIRE(N >= 1 && N < (int64_t(1) << 21), "%s: N=%lld outside [1, 2^21)", who, (long long)N);
  AVITS_REQUIRE(K >= kBlk && K < (int64_t(1) << 21) && K % kBlk == 0, "%s: K=%lld must be a multiple of 32 in [32, 2^21)", who,
                (long long)K);
  AVITS_REQUIRE(scale_groups(K) * scale_rows(std::max(M, N)) * 2 < (int64_t(1) << 31),
                "%s: %lld x %lld has 2^31 scales or more", who, (long long)std::max(M, N), (long long)K);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  return AVITS_OK;
}

template <typename T>
void run_product(const Mx4Args& a, hipStream_t s) {
  TimedLaunch timed("mxfp4_linear", s);
  auto grid = [&](int tm, int tn) {
    return dim3(unsigned(std::min<int64_t>(ceil_div64(a.M, 16 * tm) * ceil_div64(a.N, 16 * tn), 1 << 22)));
  };
  if (a.M <= 16) hipLaunchKernelGGL((mx4_rows_kernel<1, 2, T>), grid(1, 2), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((mx4_rows_kernel<4, 4, T>), grid(4, 4), dim3(256), 0, s, a);
}

// Scratch of the input gradient: the weight transposed in dtype, dy widened where
// its rows are not whole contraction tiles, and split sums of the product.
struct BackPlan {
  int64_t ld;
  size_t wt, dy, part;
};
BackPlan plan_back(int64_t M, int64_t N, int64_t K, int dtype) {
  const size_t z = dtype == AVITS_BF16 ? 2 : 4;
  BackPlan p;
  p.ld = ceil_div64(N, 64) * 64;
  p.wt = align_up(size_t(K) * size_t(p.ld) * z, 256);
  p.dy = p.ld != N ? align_up(size_t(M) * size_t(p.ld) * z, 256) : 0;
  p.part = dtype == AVITS_BF16 ? std::min<size_t>(gemm_partial_reserve(M, K), size_t(64) << 20) : 0;
  return p;
}

template <typename T>
int run_back(const void* dy, int64_t M, int64_t N, const uint8_t* wq, const uint8_t* ws, int64_t K, int dtype, void* dx,
             char* scratch, hipStream_t s) {
  const BackPlan p = plan_back(M, N, K, dtype);
  T* wt = reinterpret_cast<T*>(scratch);
  {
    TimedLaunch timed("mxfp4_transpose", s);
    hipLaunchKernelGGL(transpose4_kernel<T>, dim3(unsigned(p.ld / 64), unsigned(ceil_div64(K, 64))), dim3(256), 0, s, wq, ws, N,
                       K, wt, p.ld);
    if (p.dy) {
      T* wide = reinterpret_cast<T*>(scratch + p.wt);
      hipLaunchKernelGGL(widen_kernel<T>, dim3(unsigned(std::min<int64_t>(M, 4096)), unsigned(ceil_div64(p.ld, 256))), dim3(256),
                         0, s, static_cast<const T*>(dy), M, N, wide, p.ld);
      dy = wide;
    }
  }
  GemmArgs g{};
  g.nprob = 1;
  g.N = K;
  g.K = p.ld;
  g.n_split = g.n_split2 = K;
  g.mode0 = g.mode1 = g.mode2 = EPI_STORE;
  GemmProblem& q = g.p[0];
  q.A = dy; q.lda = p.ld; q.W = wt; q.M = M;
  q.out0 = dx; q.ld0 = K;
  return launch_gemm(g, dtype, s, "mxfp4_backward", p.part ? reinterpret_cast<float*>(scratch + p.wt + p.dy) : nullptr, p.part);
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" size_t avits_mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (check_product("mxfp4_linear_workspace_bytes", M, N, K, AVITS_BF16) != AVITS_OK) return 0;
  return 0;
}

extern "C" int avits_mxfp4_linear(const uint8_t* xq, const uint8_t* xs, int64_t M, int64_t K, const uint8_t* wq,
                                  const uint8_t* ws, const void* b, int64_t N, int32_t B, const int64_t* off,
                                  const void* gate, int64_t mod_stride, const void* resid, int dtype, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_product("mxfp4_linear", M, N, K, dtype);
  Mx4Args a = {xq, xs, wq, ws, b, gate, resid, out, M, N, K, {}};
  if (rc == AVITS_OK) rc = fill_images("mxfp4_linear", M, B, off, mod_stride, a.im);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE((gate != nullptr) == (resid != nullptr), "mxfp4_linear: gate and resid go together");
  AVITS_REQUIRE(xq && xs && wq && ws && out, "mxfp4_linear: null xq/xs/wq/ws/out");
  AVITS_REQUIRE(aligned_to({xq, xs, wq, ws, out, resid}, 16), "mxfp4_linear: xq, xs, wq, ws, resid and out must be 16-byte aligned");
  AVITS_REQUIRE(aligned_to({b, gate}, dtype == AVITS_BF16 ? 2 : 4), "mxfp4_linear: b or gate is not aligned to its element");
  const size_t need = avits_mxfp4_linear_workspace_bytes(M, N, K);
  if (need && (!workspace || workspace_bytes < need))
    return set_error(AVITS_ERR_WORKSPACE, "mxfp4_linear: workspace of %zu bytes, need %zu", workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == AVITS_BF16) run_product<bf16_t>(a, s);
  else run_product<float>(a, s);
  return launch_status("mxfp4_linear");
}

extern "C" size_t avits_mxfp4_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int dtype) {
  if (check_product("mxfp4_linear_backward_workspace_bytes", M, N, K, dtype) != AVITS_OK) return 0;
  const BackPlan p = plan_back(M, N, K, dtype);
  return p.wt + p.dy + p.part;
}

extern "C" int avits_mxfp4_linear_backward(const void* dy, int64_t M, int64_t N, const uint8_t* wq, const uint8_t* ws,
                                           int64_t K, int dtype, void* dx, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  int rc = check_product("mxfp4_linear_backward", M, N, K, dtype);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE(dy && wq && ws && dx, "mxfp4_linear_backward: null dy/wq/ws/dx");
  AVITS_REQUIRE(aligned_to({dy, wq, ws, dx}, 16), "mxfp4_linear_backward: dy, wq, ws and dx must be 16-byte aligned");
  const size_t need = avits_mxfp4_linear_backward_workspace_bytes(M, N, K, dtype);
  if (!workspace || workspace_bytes < need)
    return set_error(AVITS_ERR_WORKSPACE, "mxfp4_linear_backward: workspace of %zu bytes, need %zu", workspace_bytes, need);
  AVITS_REQUIRE(aligned_to({workspace}, 16), "mxfp4_linear_backward: workspace must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* scratch = static_cast<char*>(workspace);
  rc = dtype == AVITS_BF16 ? run_back<bf16_t>(dy, M, N, wq, ws, K, dtype, dx, scratch, s)
                           : run_back<float>(dy, M, N, wq, ws, K, dtype, dx, scratch, s);
  return rc != AVITS_OK ? rc : launch_status("mxfp4_linear_backward");
}
