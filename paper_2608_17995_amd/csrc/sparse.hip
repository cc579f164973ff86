// Attention over chosen key blocks and its backward pass: fp32, and the plans,
// checks and entry points of both types.
//
// For a query row i of head h and the keys j of the blocks that its query block keeps:
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and from do, with delta_i = do_i . o_i and p_ij = exp(s_ij - lse_i),
//   ds_ij = p_ij (do_i . v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,
//   dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i.
// A row whose block keeps nothing has o = 0 and lse = -inf.
//
// No sum crosses workgroups in a varying order: dq is made by the owners of the
// query rows, dk and dv by the owners of the key blocks (which walk the mask's
// columns), at the price of making the probabilities twice.
#include "sparse_plan.h"

namespace avits {
namespace {

// ---------------------------------------------------------------------------
// fp32, on v_mfma_f32_16x16x4_f32.  A workgroup owns 64 query rows (half a query block), 16 to a
// wave; key tiles of 64 rows pass through LDS.  Products are
// transposed (S^T = K Q^T, O^T = V^T P^T): lane l holds query row l % 16, register r
// key 4 (l / 16) + r, so the probabilities are the second product's operand as they stand.
constexpr int kFT = 64;  // rows to a tile

template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const f32x4*>(p);
  } else {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                 __uint_as_float(w[1] & 0xffff0000u)};
  }
}
__device__ __forceinline__ void store4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }

// Tiles of rows [row, row + 64) of a head of two tensors, rows from `end` on as zeros: on their way in
// registers while the tiles before them are worked on, then in LDS.
template <int DH>
struct NextTiles {
  static constexpr int kQ = DH / 4, kP = DH + 4, kN = kFT * kQ / 256;
  f32x4 x[kN], y[kN];
  __device__ __forceinline__ void fetch(const float* a, int64_t a_ld, const float* b, int64_t b_ld, int row, int end) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int e = threadIdx.x + 256 * i, r = row + e / kQ, c = 4 * (e % kQ);
      x[i] = y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r < end) {
        x[i] = load4(a + int64_t(r) * a_ld + c);
        y[i] = load4(b + int64_t(r) * b_ld + c);
      }
    }
  }
  __device__ __forceinline__ void put(float* a, float* b) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int e = threadIdx.x + 256 * i, at = e / kQ * kP + 4 * (e % kQ);
      store4(a + at, x[i]);
      store4(b + at, y[i]);
    }
  }
};

// 16 rows' fragments in registers: lane l has row l % 16, elements 16 j + 4 (l / 16) + e.
template <int DH>
__device__ __forceinline__ void load_rows(f32x4* f, const float* src, int64_t ld, int row, int end) {
  const int lane = threadIdx.x % kWave, r = row + lane % 16;
#pragma unroll
  for (int j = 0; j < DH / 16; ++j)
    f[j] = r < end ? load4(src + int64_t(r) * ld + 16 * j + 4 * (lane / 16)) : f32x4{0.f, 0.f, 0.f, 0.f};
}

// sum over d of tile[row0 + lane % 16][d] f[d]: 16 rows of an LDS tile against 16 register rows.
template <int DH>
__device__ __forceinline__ f32x4 rows_product(const float* tile, int row0, const f32x4* f) {
  constexpr int kP = DH + 4;
  const int lane = threadIdx.x % kWave;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < DH / 16; ++j) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(tile + (row0 + lane % 16) * kP + 16 * j + 4 * (lane / 16));
#pragma unroll
    for (int e = 0; e < 4; ++e) s = mfma16x16x4(t[e], f[j][e], s);
  }
  return s;
}

// acc[dt] += tile^T p over the 16 tile rows from row0: p's register r is tile row row0 + 4 (lane / 16) + r.
template <int DH>
__device__ __forceinline__ void columns_product(const float* tile, int row0, const f32x4& p, f32x4* acc) {
  constexpr int kP = DH + 4;
  const int lane = threadIdx.x % kWave;
  const float* src = tile + (row0 + 4 * (lane / 16)) * kP + lane % 16;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int dt = 0; dt < DH / 16; ++dt) acc[dt] = mfma16x16x4(src[r * kP + 16 * dt], p[r], acc[dt]);
}

__device__ __forceinline__ float quad_max(float v) { return max_xor32(fmaxf(v, __shfl_xor(v, 16))); }
__device__ __forceinline__ float quad_sum(float v) { return sum_xor32(v + __shfl_xor(v, 16)); }

// The sums of a workgroup's waves over the same 16 rows: each wave's to LDS, then (the caller waits between)
// elements c .. c + 3 of row i added up in the waves' order.
template <int DH>
__device__ __forceinline__ void put_sums(float* to, int wave, const f32x4* acc) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int d = 0; d < DH / 16; ++d) store4(to + (16 * wave + lane % 16) * (DH + 4) + 16 * d + 4 * (lane / 16), acc[d]);
}
template <int DH>
__device__ __forceinline__ f32x4 add_sums(const float* from, int i, int c) {
  f32x4 v = load4(from + i * (DH + 4) + c);
#pragma unroll
  for (int p = 1; p < 4; ++p) v += load4(from + (16 * p + i) * (DH + 4) + c);
  return v;
}

// The forward pass: bound by the fp32 matrix instructions (4096 rows of 16 heads of 128, half the blocks kept: 774 us, 89 TFLOP/s
// of the 154 of a large library product), for few rows by the latency of a tile's two barriers and products (288 rows of 4 heads
// of 64: 11 us for five tiles in a row; without SPLIT 25).  SPLIT, for few rows: a workgroup owns 16 of them, each of its waves a quarter of every
// tile's keys, and the waves' maxima and sums meet in LDS at the end.
template <int DH, bool SPLIT>
__global__ __launch_bounds__(256, 2) void sparse_f32_kernel(const SparseArgs a) {
  constexpr int kP = DH + 4, kD = DH / 16, kQ = DH / 4, kT = SPLIT ? 1 : 4, kRows = SPLIT ? 16 : 64;
  __shared__ __attribute__((aligned(16))) float kt[kFT * kP], vt[kFT * kP];
  __shared__ float top[4][16], sum[4][16];
  const int blk = blockIdx.x / (kQB / kRows), h = blockIdx.y, lane = threadIdx.x % kWave;
  const Seq s = seq_of<false>(a.seq, blk);
  const int wave = threadIdx.x / kWave, first = s.q_lo + (blk - s.qb) * kQB + kRows * (blockIdx.x % (kQB / kRows));
  if (first >= s.q_hi) return;
  const int row = first + (SPLIT ? 0 : 16 * wave) + lane % 16, key0 = SPLIT ? 16 * wave : 0;
  const float* K = static_cast<const float*>(a.k) + int64_t(h / a.group) * DH;
  const float* V = static_cast<const float*>(a.v) + int64_t(h / a.group) * DH;
  f32x4 q[kD], o[kD];
  NextTiles<DH> ahead;
  auto fetch = [&](int j) { ahead.fetch(K, a.k_ld, V, a.v_ld, s.k_lo + j * kKB, s.k_hi); };
  BlockWalk walk(a, h, blk, s.nk);
  int j = walk.next();
  if (j >= 0) fetch(j);
  load_rows<DH>(q, static_cast<const float*>(a.q) + int64_t(h) * DH, a.q_ld, row - lane % 16, s.q_hi);
#pragma unroll
  for (int d = 0; d < kD; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  while (j >= 0) {
    __syncthreads();
    ahead.put(kt, vt);
    const int n = s.k_hi - (s.k_lo + j * kKB);
    j = walk.next();
    if (j >= 0) fetch(j);
    __syncthreads();
    f32x4 x[kT];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      x[t] = rows_product<DH>(kt, key0 + 16 * t, q);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[t][r] = key0 + 16 * t + 4 * (lane / 16) + r < n ? x[t][r] * a.scale : -INFINITY;
        mx = fmaxf(mx, x[t][r]);
      }
    }
    mx = fmaxf(m, quad_max(mx));
    const float ref = mx == -INFINITY ? 0.f : mx, corr = expf(m - ref);
    m = mx;
    l *= corr;
#pragma unroll
    for (int d = 0; d < kD; ++d) o[d] *= corr;
#pragma unroll
    for (int t = 0; t < kT; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[t][r] = expf(x[t][r] - ref);
        l += x[t][r];
      }
      columns_product<DH>(vt, key0 + 16 * t, x[t], o);
    }
  }
  l = quad_sum(l);
  const bool none = walk.total == 0;
  if constexpr (SPLIT) {
    const int r = lane % 16;
    if (lane < 16) top[wave][r] = m;
    __syncthreads();  // also: the tiles are done with
    m = fmaxf(fmaxf(top[0][r], top[1][r]), fmaxf(top[2][r], top[3][r]));
    const float w = expf(top[wave][r] - (m == -INFINITY ? 0.f : m));
    if (lane < 16) sum[wave][r] = l * w;
#pragma unroll
    for (int d = 0; d < kD; ++d) o[d] *= w;
    put_sums<DH>(kt, wave, o);
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * kQ; e += 256) {
      const int i = e / kQ, c = 4 * (e % kQ), to = first + i;
      if (to >= s.q_hi) return;
      const float den = sum[0][i] + sum[1][i] + sum[2][i] + sum[3][i];
      if (a.lse && c == 0)
        a.lse[int64_t(h) * a.M + to] =
            none ? -INFINITY : fmaxf(fmaxf(top[0][i], top[1][i]), fmaxf(top[2][i], top[3][i])) + logf(den);
      store4(static_cast<float*>(a.o) + int64_t(to) * a.o_ld + int64_t(h) * DH + c, none ? f32x4{0.f, 0.f, 0.f, 0.f} : add_sums<DH>(kt, i, c) / den);
    }
  } else {
    if (row >= s.q_hi) return;
    if (a.lse && lane < 16) a.lse[int64_t(h) * a.M + row] = none ? -INFINITY : m + logf(l);
    float* dst = static_cast<float*>(a.o) + int64_t(row) * a.o_ld + int64_t(h) * DH + 4 * (lane / 16);
#pragma unroll
    for (int d = 0; d < kD; ++d) store4(dst + 16 * d, none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[d] / l);
  }
}

template <int DH, bool SPLIT>
__global__ __launch_bounds__(256, 2) void sparse_dq_f32_kernel(const SparseArgs a) {
  constexpr int kP = DH + 4, kD = DH / 16, kQ = DH / 4, kT = SPLIT ? 1 : 4, kRows = SPLIT ? 16 : 64;
  __shared__ __attribute__((aligned(16))) float kt[kFT * kP], vt[kFT * kP];
  const int blk = blockIdx.x / (kQB / kRows), h = blockIdx.y, lane = threadIdx.x % kWave;
  const Seq s = seq_of<false>(a.seq, blk);
  const int wave = threadIdx.x / kWave, first = s.q_lo + (blk - s.qb) * kQB + kRows * (blockIdx.x % (kQB / kRows));
  if (first >= s.q_hi) return;
  const int row = first + (SPLIT ? 0 : 16 * wave) + lane % 16, key0 = SPLIT ? 16 * wave : 0;
  const float* K = static_cast<const float*>(a.k) + int64_t(h / a.group) * DH;
  const float* V = static_cast<const float*>(a.v) + int64_t(h / a.group) * DH;
  f32x4 q[kD], g[kD], dq[kD];
  NextTiles<DH> ahead;
  auto fetch = [&](int j) { ahead.fetch(K, a.k_ld, V, a.v_ld, s.k_lo + j * kKB, s.k_hi); };
  BlockWalk walk(a, h, blk, s.nk);
  int j = walk.next();
  if (j >= 0) fetch(j);
  load_rows<DH>(q, static_cast<const float*>(a.q) + int64_t(h) * DH, a.q_ld, row - lane % 16, s.q_hi);
  load_rows<DH>(g, static_cast<const float*>(a.dout) + int64_t(h) * DH, a.do_ld, row - lane % 16, s.q_hi);
#pragma unroll
  for (int d = 0; d < kD; ++d) dq[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float2 st = row < s.q_hi ? a.stats[int64_t(h) * a.M + row] : make_float2(INFINITY, 0.f);
  const float lse = st.x, delta = st.y;
  while (j >= 0) {
    __syncthreads();
    ahead.put(kt, vt);
    const int n = s.k_hi - (s.k_lo + j * kKB);
    j = walk.next();
    if (j >= 0) fetch(j);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      const f32x4 x = rows_product<DH>(kt, key0 + 16 * t, q), dp = rows_product<DH>(vt, key0 + 16 * t, g);
      f32x4 ds;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        ds[r] = key0 + 16 * t + 4 * (lane / 16) + r < n ? expf(x[r] * a.scale - lse) * (dp[r] - delta) : 0.f;
      columns_product<DH>(kt, key0 + 16 * t, ds, dq);
    }
  }
  const float scale = grad_scale(a, s);
  if constexpr (SPLIT) {
    __syncthreads();
    put_sums<DH>(kt, wave, dq);
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * kQ; e += 256) {
      const int i = e / kQ, c = 4 * (e % kQ);
      if (first + i >= s.q_hi) return;
      store4(static_cast<float*>(a.dq) + int64_t(first + i) * a.dq_ld + int64_t(h) * DH + c, add_sums<DH>(kt, i, c) * scale);
    }
  } else {
    if (row >= s.q_hi) return;
    float* dst = static_cast<float*>(a.dq) + int64_t(row) * a.dq_ld + int64_t(h) * DH + 4 * (lane / 16);
#pragma unroll
    for (int d = 0; d < kD; ++d) store4(dst + 16 * d, dq[d] * scale);
  }
}

// dk and dv of a key block: 16 keys to a wave, the query rows that keep the block pass through LDS, 64 at a time.
// SPLIT: a quarter of the block to a workgroup, a quarter of every 64 rows to each wave.
// Two workgroups to a CU, though 256 registers leave 36 bytes of scratch at heads of 128 (4096 rows of
// 16 heads, 30 % kept: the pass 1620 us, with one workgroup and no scratch 1840).
template <int DH, bool SPLIT>
__global__ __launch_bounds__(256, 2) void sparse_dkv_f32_kernel(const SparseArgs a) {
  constexpr int kP = DH + 4, kD = DH / 16, kQ = DH / 4, kT = SPLIT ? 1 : 4;
  __shared__ __attribute__((aligned(16))) float qt[kFT * kP], gt[kFT * kP];
  __shared__ float ls[kFT], dl[kFT];
  const int blk = SPLIT ? blockIdx.x / 4 : blockIdx.x, hk = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Seq s = seq_of<true>(a.seq, blk);
  const int first = s.k_lo + (blk - s.kb) * kKB + 16 * (SPLIT ? blockIdx.x % 4 : wave), row0 = SPLIT ? 16 * wave : 0;
  if (SPLIT && first >= s.k_hi) return;
  f32x4 k[kD], v[kD], dk[kD], dv[kD];
  const int nq = (s.q_hi - s.q_lo + kQB - 1) / kQB;
  // The next 64 rows of a query block that keeps this key block.
  int h = hk * a.group, i = -1, row = -1;
  auto next = [&]() {
    if (row >= 0 && row + kFT < std::min(s.q_hi, s.q_lo + (i + 1) * kQB)) {
      row += kFT;
      return true;
    }
    for (; h < (hk + 1) * a.group; ++h, i = -1)
      while (++i < nq)
        if (kept(a, h, s.qb + i, blk - s.kb)) {
          row = s.q_lo + i * kQB;
          return true;
        }
    return false;
  };
  NextTiles<DH> ahead;
  float2 st;
  auto fetch = [&]() {
    ahead.fetch(static_cast<const float*>(a.q) + int64_t(h) * DH, a.q_ld, static_cast<const float*>(a.dout) + int64_t(h) * DH, a.do_ld, row, s.q_hi);
    const int r = row + threadIdx.x % kFT;
    st = r < s.q_hi ? a.stats[int64_t(h) * a.M + r] : make_float2(INFINITY, 0.f);  // past the end: no probability
  };
  bool more = next();
  if (more) fetch();
  load_rows<DH>(k, static_cast<const float*>(a.k) + int64_t(hk) * DH, a.k_ld, first, s.k_hi);
  load_rows<DH>(v, static_cast<const float*>(a.v) + int64_t(hk) * DH, a.v_ld, first, s.k_hi);
#pragma unroll
  for (int d = 0; d < kD; ++d) dk[d] = dv[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  while (more) {
    __syncthreads();
    ahead.put(qt, gt);
    if (threadIdx.x < kFT) {
      ls[threadIdx.x] = st.x;
      dl[threadIdx.x] = st.y;
    }
    more = next();
    if (more) fetch();
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      const f32x4 x = rows_product<DH>(qt, row0 + 16 * t, k), dp = rows_product<DH>(gt, row0 + 16 * t, v);
      f32x4 p, ds;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = row0 + 16 * t + 4 * (lane / 16) + r;
        p[r] = expf(x[r] * a.scale - ls[e]);
        ds[r] = p[r] * (dp[r] - dl[e]);
      }
      columns_product<DH>(gt, row0 + 16 * t, p, dv);
      columns_product<DH>(qt, row0 + 16 * t, ds, dk);
    }
  }
  float* pk = static_cast<float*>(a.dk) + int64_t(hk) * DH;
  float* pv = static_cast<float*>(a.dv) + int64_t(hk) * DH;
  const float scale = grad_scale(a, s);
  if constexpr (SPLIT) {
    __syncthreads();
    put_sums<DH>(qt, wave, dk);
    put_sums<DH>(gt, wave, dv);
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * kQ; e += 256) {
      const int r = e / kQ, c = 4 * (e % kQ);
      if (first + r >= s.k_hi) return;
      store4(pk + int64_t(first + r) * a.dk_ld + c, add_sums<DH>(qt, r, c) * scale);
      store4(pv + int64_t(first + r) * a.dv_ld + c, add_sums<DH>(gt, r, c));
    }
  } else {
    const int to = first + lane % 16, c = 4 * (lane / 16);
    if (to >= s.k_hi) return;
#pragma unroll
    for (int d = 0; d < kD; ++d) {
      store4(pk + int64_t(to) * a.dk_ld + c + 16 * d, dk[d] * scale);
      store4(pv + int64_t(to) * a.dv_ld + c + 16 * d, dv[d]);
    }
  }
}

// delta = do . o of every row and head, beside lse: DH / 8 lanes to a head; a workgroup takes 16 rows of up to
// 64 heads, whose results pass through LDS so that they are written row after row (straight from the
// lanes, 8 bytes to a place M apart, 9.5 us at 4608 rows of 16 heads of 128; 7.4 at a copy's rate).  The first workgroups make
// the plans of dq and of dk and dv meanwhile: 10 to 11 us with that of dq.
constexpr int kDeltaRows = 16, kDeltaHeads = 64;
template <typename T, int DH>
__global__ __launch_bounds__(1024) void sparse_delta_kernel(const SparseArgs a, SparsePlan* plan_q, SparsePlan* plan_k) {
  constexpr int kL = DH / 8, kStep = 1024 / kL / kDeltaRows;  // lanes to a head, heads at once
  __shared__ int counts[kMaxUnits];
  __shared__ uint64_t sums[1024];
  __shared__ float out[kDeltaHeads][kDeltaRows + 1];
  int64_t wg = wide_block();
  if (plan_q && wg-- == 0) return sparse_plan<false, 1024>(a, plan_q, counts, sums);
  if (plan_k && wg-- == 0) return sparse_plan<true, 1024>(a, plan_k, counts, sums);
  const int chunks = (a.H + kDeltaHeads - 1) / kDeltaHeads, h0 = int(wg % chunks) * kDeltaHeads, nh = std::min(kDeltaHeads, a.H - h0);
  const int64_t row0 = wg / chunks * kDeltaRows;
  const int g = threadIdx.x / kL, c = threadIdx.x % kL * 8, r = g / kStep;
  const int64_t row = row0 + r;
  for (int hh = g % kStep; hh < nh && row < a.seq.q_row[kMaxSeqs]; hh += kStep) {  // groups of lanes leave together
    const T* x = static_cast<const T*>(a.dout) + row * a.do_ld + int64_t(h0 + hh) * DH + c;
    const T* y = static_cast<const T*>(a.o) + row * a.o_ld + int64_t(h0 + hh) * DH + c;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const f32x4 u = load4(x + e), v = load4(y + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += u[k] * v[k];
    }
    sum = group_sum(sum, kL);
    if (c == 0) out[hh][r] = sum;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nh * kDeltaRows; i += 1024) {
    const int64_t to = row0 + i % kDeltaRows, at = (h0 + i / kDeltaRows) * a.M + to;
    if (to < a.seq.q_row[kMaxSeqs]) a.stats[at] = make_float2(a.lse[at], out[i / kDeltaRows][i % kDeltaRows]);
  }
}

// 16 rows (keys) to a workgroup up to 256 workgroups of 64, one to a CU.  1024 rows of 16 heads of 128, half the
// blocks kept: 82 us, 64 to a workgroup 93; 2048 rows of 16 heads of 64, 131 and 128.
bool split(int64_t workgroups) { return workgroups <= 256; }

template <int DH>
void forward_f32(const SparseArgs& a, hipStream_t s) {
  const unsigned n = 2 * unsigned(a.seq.q_blk[a.seq.B]), heads = unsigned(a.H);
  if (split(int64_t(n) * heads)) hipLaunchKernelGGL((sparse_f32_kernel<DH, true>), dim3(4 * n, heads), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((sparse_f32_kernel<DH, false>), dim3(n, heads), dim3(256), 0, s, a);
}

template <int DH>
void backward_f32(const SparseArgs& a, hipStream_t s) {
  const unsigned nq = 2 * unsigned(a.seq.q_blk[a.seq.B]), nk = unsigned(a.seq.k_blk[a.seq.B]), H = unsigned(a.H), Hk = unsigned(a.H / a.group);
  if (nq > 0) {
    if (split(int64_t(nq) * H)) hipLaunchKernelGGL((sparse_dq_f32_kernel<DH, true>), dim3(4 * nq, H), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sparse_dq_f32_kernel<DH, false>), dim3(nq, H), dim3(256), 0, s, a);
  }
  if (nk > 0) {
    if (split(int64_t(nk) * Hk)) hipLaunchKernelGGL((sparse_dkv_f32_kernel<DH, true>), dim3(4 * nk, Hk), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sparse_dkv_f32_kernel<DH, false>), dim3(nk, Hk), dim3(256), 0, s, a);
  }
}

int fill(SparseArgs& a, const char* what, const avits_rows* q, const avits_rows* k, const avits_rows* v, int64_t M, int64_t N,
         int32_t B, const int64_t* q_off, const int64_t* k_off, int32_t H, int32_t Hk, int32_t d, const uint64_t* mask, int64_t words,
         float scale, int dtype) {
  a = SparseArgs{};
  const int rc = seq_blocks(a.seq, what, B, q_off, M, k_off, N);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(Hk >= 1 && H >= Hk && H % Hk == 0 && H <= 1024, "%s: H=%d must be a multiple of Hk=%d, at most 1024", what, H, Hk);
  if (d != 64 && d != 128) return set_error(AVITS_ERR_UNSUPPORTED, "%s: head dim %d (need 64 or 128)", what, d);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", what, dtype);
  // (The gradients start their logits from -lse / scale.)
  AVITS_REQUIRE(scale >= 0x1p-64f && scale <= 0x1p64f, "%s: scale=%g outside [2^-64, 2^64]", what, double(scale));
  int nk = 0;
  for (int b = 0; b < B; ++b) nk = std::max(nk, a.seq.k_blk[b + 1] - a.seq.k_blk[b]);
  AVITS_REQUIRE(!mask || (words >= (nk + 63) / 64 && words < (int64_t(1) << 20)), "%s: %lld words a row for %d key blocks", what,
                (long long)words, nk);
  AVITS_REQUIRE(reinterpret_cast<uintptr_t>(mask) % 8 == 0, "%s: the mask is not aligned to its words", what);
  AVITS_REQUIRE(q && k && v, "%s: null rows", what);
  // A workgroup of 256 to each query block of a head; fp32: two to each query block, heads along y.
  if (!fits_x(dtype == AVITS_BF16 ? int64_t(a.seq.q_blk[B]) * H : 2 * int64_t(a.seq.q_blk[B]), 256))
    return set_error(AVITS_ERR_UNSUPPORTED, "%s: %d query blocks of %d heads", what, a.seq.q_blk[B], H);
  a.q = q->p, a.k = k->p, a.v = v->p;
  a.q_ld = q->ld, a.k_ld = k->ld, a.v_ld = v->ld;
  a.mask = mask;
  a.words = words;
  a.M = M;
  a.H = H;
  a.group = H / Hk;
  a.d = d;
  a.scale = scale;
  a.seq.q_row[kMaxSeqs] = a.seq.q_row[B];
  a.seq.q_blk[kMaxSeqs] = a.seq.q_blk[B];
  a.seq.k_blk[kMaxSeqs] = a.seq.k_blk[B];
  return AVITS_OK;
}

// Rows of `heads` heads: there (unless there are none), on 16 bytes and apart.
int check_rows(const char* what, const char* name, const avits_rows* r, int64_t rows, int64_t heads, int d, int dtype) {
  if (rows == 0) return AVITS_OK;
  AVITS_REQUIRE(r && r->p, "%s: null %s", what, name);
  const int64_t elem = dtype == AVITS_BF16 ? 2 : 4;
  AVITS_REQUIRE(reinterpret_cast<uintptr_t>(r->p) % 16 == 0 && (rows == 1 || r->ld * elem % 16 == 0),
                "%s: the rows of %s must lie on 16 bytes (row stride %lld)", what, name, (long long)r->ld);
  AVITS_REQUIRE(rows == 1 || (r->ld >= heads * d && r->ld < (int64_t(1) << 24)), "%s: row stride %lld of %s (heads * d to 2^24)", what,
                (long long)r->ld, name);
  return AVITS_OK;
}

#define AVITS_ROWS(name, rows, heads)                                                   \
  do {                                                                                  \
    const int rc_ = check_rows(what, #name, name, rows, heads, d, dtype);               \
    if (rc_ != AVITS_OK) return rc_;                                                    \
  } while (0)

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 4096;

// Bytes of a slot of a query block's (max, sum) and outputs.
size_t slot_bytes(int32_t d) { return size_t(kQB) * size_t(d + 2) * sizeof(float); }
size_t plan_bytes() { return align_up(sizeof(SparsePlan), 256); }

// Whether a plan cuts the lists of so many units: not short ones, for which the launches cost more (1000 rows of 16 heads of 64,
// half kept: 16 us, with a plan 22).
bool planned(int64_t units, int64_t most, bool mask) {
  return mask && units > kFewUnits && units <= kMaxUnits && most > 2 * kMinList;
}
// A side of a backward pass: with few units also without a mask (4096 rows of one head, all kept: 158 -> 73 us).
bool planned_backward(int64_t units, int64_t most, bool mask) {
  return units > kFewUnits ? planned(units, most, mask) : units > 0 && most > 2 * kMinList;
}

// What the forward pass of `units` units with lists of at most `most` blocks needs.
size_t forward_bytes(int64_t units, int64_t most, int32_t d, bool mask) {
  if (planned(units, most, mask)) return plan_bytes() + size_t(sparse_slots(units, most)) * slot_bytes(d);
  const int p = sparse_pieces(units, most);
  return p > 1 ? size_t(p) * size_t(units) * slot_bytes(d) : 0;
}

// One side of a backward pass, for up to so many units.
size_t side_bytes(int64_t units, int64_t most, int32_t d) {
  return plan_bytes() + size_t(sparse_slots(std::min<int64_t>(units, kMaxUnits), most)) * kQB * d * sizeof(float);
}

size_t stats_bytes(int64_t M, int32_t H) { return align_up(size_t(M) * size_t(H) * sizeof(float2), 256); }

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" size_t avits_sparse_attention_workspace_bytes(int64_t M, int64_t N, int32_t B, int32_t H, int32_t d, int dtype) {
  if (M < 0 || N < 0 || M >= kMaxRows || N >= kMaxRows || B < 1 || B > kMaxSeqs || H < 1 || H > 1024 || (d != 64 && d != 128)) return 0;
  if (dtype != AVITS_BF16) return 0;
  size_t most = 0;  // fewer rows, or fewer sequences, may need more
  for (int64_t blocks = 1; blocks <= ceil_div64(M, kQB) + B && blocks * H <= kMaxUnits; ++blocks)
    for (bool mask : {false, true}) most = std::max(most, forward_bytes(blocks * H, ceil_div64(N, kKB), d, mask));
  return most;
}

extern "C" int avits_sparse_attention(const avits_rows* q, const avits_rows* k, const avits_rows* v, int64_t M, int64_t N, int32_t B,
                                      const int64_t* q_off, const int64_t* k_off, int32_t H, int32_t Hk, int32_t d,
                                      const uint64_t* mask, int64_t words, float scale, int dtype, const avits_rows* o, float* lse,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "sparse_attention";
  SparseArgs a;
  const int rc = fill(a, what, q, k, v, M, N, B, q_off, k_off, H, Hk, d, mask, words, scale, dtype);
  if (rc != AVITS_OK) return rc;
  const int64_t m = a.seq.q_row[B], n = a.seq.k_row[B];
  AVITS_ROWS(q, m, H);
  AVITS_ROWS(k, n, Hk);
  AVITS_ROWS(v, n, Hk);
  AVITS_ROWS(o, m, H);
  if (m == 0) return AVITS_OK;
  a.o = o->p;
  a.o_ld = o->ld;
  a.lse = lse;
  a.pieces = 1;
  if (dtype == AVITS_BF16) {
    int most = 0;
    for (int b = 0; b < B; ++b) most = std::max(most, a.seq.k_blk[b + 1] - a.seq.k_blk[b]);
    const int64_t units = int64_t(a.seq.q_blk[B]) * H;
    const size_t need = forward_bytes(units, most, d, mask != nullptr);
    if (need > 0) {
      if (!workspace || workspace_bytes < need)
        return set_error(AVITS_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : size_t(0), need);
      AVITS_REQUIRE(reinterpret_cast<uintptr_t>(workspace) % 16 == 0, "%s: the workspace is not 16-byte aligned", what);
    }
    char* at = static_cast<char*>(workspace);
    if (planned(units, most, mask != nullptr)) {
      a.slots = sparse_slots(units, most);
      a.plan = reinterpret_cast<const SparsePlan*>(at);
      at += plan_bytes();
    } else {
      a.pieces = sparse_pieces(units, most);
      a.slots = a.pieces > 1 ? units * a.pieces : 0;
    }
    a.part = reinterpret_cast<float*>(at);
    a.part_ml = a.part + a.slots * kQB * d;
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  TimedLaunch timed(what, s);
  if (dtype == AVITS_F32) d == 128 ? forward_f32<128>(a, s) : forward_f32<64>(a, s);
  else launch_sparse_bf16(a, s);
  return launch_status(what);
}

extern "C" size_t avits_sparse_attention_backward_workspace_bytes(int64_t M, int64_t N, int32_t B, int32_t H, int32_t Hk, int32_t d, int dtype) {
  if (M < 0 || N < 0 || M >= kMaxRows || N >= kMaxRows || B < 1 || B > kMaxSeqs || H < 1 || H > 1024 || Hk < 1 || H % Hk != 0 || (d != 64 && d != 128)) return 0;
  size_t most = stats_bytes(M, H);
  if (dtype != AVITS_BF16) return most;
  const int64_t nq = ceil_div64(M, kQB) + B, nk = ceil_div64(N, kKB) + B;  // blocks, at most
  return most + side_bytes(nq * H, nk, d) + side_bytes(nk * Hk, nq * (H / Hk), d);
}

extern "C" int avits_sparse_attention_backward(const avits_rows* dout, const avits_rows* q, const avits_rows* k, const avits_rows* v,
                                               const avits_rows* o, const float* lse, int64_t M, int64_t N, int32_t B,
                                               const int64_t* q_off, const int64_t* k_off, int32_t H, int32_t Hk, int32_t d,
                                               const uint64_t* mask, int64_t words, float scale, int dtype, const avits_rows* dq,
                                               const avits_rows* dk, const avits_rows* dv, void* workspace, size_t workspace_bytes,
                                               void* stream) {
  const char* what = "sparse_attention_backward";
  SparseArgs a;
  const int rc = fill(a, what, q, k, v, M, N, B, q_off, k_off, H, Hk, d, mask, words, scale, dtype);
  if (rc != AVITS_OK) return rc;
  const int64_t m = a.seq.q_row[B], n = a.seq.k_row[B];
  AVITS_ROWS(q, m, H);
  AVITS_ROWS(k, n, Hk);
  AVITS_ROWS(v, n, Hk);
  AVITS_ROWS(o, m, H);
  AVITS_ROWS(dout, m, H);
  AVITS_ROWS(dq, m, H);
  AVITS_ROWS(dk, n, Hk);
  AVITS_ROWS(dv, n, Hk);
  if (m == 0 && n == 0) return AVITS_OK;
  AVITS_REQUIRE(lse || m == 0, "%s: null lse", what);
  // A workgroup of 512 to each key block of a head; fp32: of 256 to each key block, heads along y.
  if (!(dtype == AVITS_BF16 ? fits_x(int64_t(a.seq.k_blk[B]) * Hk, 512) : fits_x(a.seq.k_blk[B], 256)))
    return set_error(AVITS_ERR_UNSUPPORTED, "%s: %d key blocks of %d heads", what, a.seq.k_blk[B], Hk);
  const size_t need = avits_sparse_attention_backward_workspace_bytes(M, N, B, H, Hk, d, dtype);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return set_error(AVITS_ERR_WORKSPACE, "%s: workspace of %zu bytes, need %zu", what, workspace ? workspace_bytes : size_t(0), need);
  AVITS_REQUIRE(reinterpret_cast<uintptr_t>(workspace) % 16 == 0, "%s: the workspace is not 16-byte aligned", what);
  if (m > 0) {
    a.dout = dout->p, a.o = o->p, a.dq = dq->p;
    a.do_ld = dout->ld, a.o_ld = o->ld, a.dq_ld = dq->ld;
  }
  if (n > 0) {
    a.dk = dk->p, a.dv = dv->p;
    a.dk_ld = dk->ld, a.dv_ld = dv->ld;
  }
  a.lse = const_cast<float*>(lse);
  a.stats = static_cast<float2*>(workspace);
  a.pieces = 1;
  // The plans of dq and of dk and dv, and their slots.
  SparseArgs ak = a;
  SparsePlan *plan_q = nullptr, *plan_k = nullptr;
  if (dtype == AVITS_BF16 && m > 0 && n > 0) {
    int most_q = 0, most_k = 0;
    for (int b = 0; b < B; ++b) {
      most_q = std::max(most_q, a.seq.k_blk[b + 1] - a.seq.k_blk[b]);
      most_k = std::max(most_k, (a.seq.q_blk[b + 1] - a.seq.q_blk[b]) * a.group);
    }
    char* at = static_cast<char*>(workspace) + stats_bytes(M, H);
    const int64_t uq = int64_t(a.seq.q_blk[B]) * H, uk = int64_t(a.seq.k_blk[B]) * Hk;
    if (planned_backward(uq, most_q, mask != nullptr)) {
      a.plan = plan_q = reinterpret_cast<SparsePlan*>(at);
      a.slots = sparse_slots(uq, most_q);
      a.part = reinterpret_cast<float*>(at + plan_bytes());
      at += plan_bytes() + size_t(a.slots) * kQB * d * sizeof(float);
    }
    if (planned_backward(uk, most_k, mask != nullptr)) {
      ak.plan = plan_k = reinterpret_cast<SparsePlan*>(at);
      ak.slots = sparse_slots(uk, most_k);
      ak.part = reinterpret_cast<float*>(at + plan_bytes());
    }
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  TimedLaunch timed(what, s);
  if (m > 0) {
    const dim3 grid = wide_grid(ceil_div64(m, kDeltaRows) * ceil_div64(H, kDeltaHeads) + (plan_q != nullptr) + (plan_k != nullptr));
    if (dtype == AVITS_BF16) {
      if (d == 128) hipLaunchKernelGGL((sparse_delta_kernel<bf16_t, 128>), grid, dim3(1024), 0, s, a, plan_q, plan_k);
      else hipLaunchKernelGGL((sparse_delta_kernel<bf16_t, 64>), grid, dim3(1024), 0, s, a, plan_q, plan_k);
    } else {
      if (d == 128) hipLaunchKernelGGL((sparse_delta_kernel<float, 128>), grid, dim3(1024), 0, s, a, plan_q, plan_k);
      else hipLaunchKernelGGL((sparse_delta_kernel<float, 64>), grid, dim3(1024), 0, s, a, plan_q, plan_k);
    }
  }
  if (dtype == AVITS_F32) d == 128 ? backward_f32<128>(a, s) : backward_f32<64>(a, s);
  else launch_sparse_back_bf16(a, ak, s);
  return launch_status(what);
}
