// Backward pass of the attention over chosen key blocks in bf16, on v_mfma_f32_32x32x16_bf16.
//
// dq: a workgroup owns a query block of 128 rows of a head and walks the set bits of its mask row;
// dk, dv: a workgroup owns a key block of 64 rows and walks the query blocks of its key head's query
// heads that keep it.  Both make the logits and probabilities again from lse, so seven
// products run where five would do, and no sum crosses workgroups.
//
// What bounds such kernels is the LDS: a 32x32x16 product takes 32 cycles of a SIMD and its LDS operand
// 8 cycles of the CU's LDS, all of it with four SIMDs.  So each wave covers 64 x 32 rows and keys: one
// fragment feeds two products, at one wave to a SIMD with all its registers (the other operands
// and the sums stay in them).
// Probabilities and ds are rounded to bf16 for the second products, which the matrix instruction
// takes; everything else is fp32.
#include "sparse_attn.h"

namespace avits {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x16 mfma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Position of 16-byte chunk c of row r of an LDS tile is c ^ swz(r): reads of one chunk of 16 rows, and
// of four chunks of four rows (the transposed ones), touch every bank once.
template <int DH>
__device__ __forceinline__ int swz(int r) {
  return DH == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

// Byte address within a tile of the fragment of rows row0 + l % 32, elements 16 c + 8 (l / 32) ..
template <int DH>
struct Frag {
  int row_at, tr_at;
  __device__ __forceinline__ Frag() {
    const int lane = threadIdx.x % kWave, l32 = lane % 32, hi = lane / 32;
    row_at = l32 * (DH * 2) + (hi ^ swz<DH>(l32)) * 16;
    const int r = (lane % 16) / 4 + 4 * hi;
    tr_at = r * (DH * 2) + ((2 * ((lane / 16) % 2) + (lane % 4) / 2) ^ swz<DH>(r)) * 16 + (lane % 2) * 8;
  }
  // Keeps the fragments' addresses from being made once for all steps, which costs registers.
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row_at), "+v"(tr_at)); }
  __device__ __forceinline__ bf16x8 rows(const char* tile, int c) const {
    return as_bf16x8(*reinterpret_cast<const u32x4*>(tile + (row_at ^ (32 * c))));
  }
  // Column 32 dt + l % 32 of rows 16 c + 4 (l / 32) + {0 .. 3, 8 .. 11}: the order of a product's registers.
  __device__ __forceinline__ bf16x8 columns(const char* tile, int c, int dt) const {
    const char* p = tile + 16 * c * (DH * 2);
    const u32x2 lo = lds_read_tr(p + (tr_at ^ (64 * dt))), up = lds_read_tr(p + 8 * (DH * 2) + (tr_at ^ (64 * dt) ^ 32));
    return as_bf16x8(u32x4{lo[0], lo[1], up[0], up[1]});
  }
};

// Registers r - 1 and r (odd) of a product into their chunk of the next product's operand.
__device__ __forceinline__ void put(bf16x8& chunk, int r, float lo, float up) {
  u32x4 v = __builtin_bit_cast(u32x4, chunk);
  v[(r % 8) / 2] = pack_bf2(lo, up);
  chunk = as_bf16x8(v);
}

// Byte offsets of one load instruction's lanes: rows of DH elements, 1 KB to an instruction.
template <int DH>
__device__ __forceinline__ uint32_t load_off(int i, int64_t ld) {
  constexpr int kCH = DH / 8, kR = kWave / kCH;
  const int lane = threadIdx.x % kWave, r = kR * i + lane / kCH;
  return uint32_t(r) * uint32_t(ld * 2) + uint32_t(((lane % kCH) ^ swz<DH>(r)) * 16);
}

// Buffer over rows [first, end) of a head: what lies behind reads as zeros.
__device__ __forceinline__ u32x4 rows_rsrc(const bf16_t* base, int64_t ld, int first, int end, int width) {
  const int64_t bytes = end > first ? (int64_t(end - first - 1) * ld + width) * 2 : 0;
  u32x4 r = buffer_rsrc(base + int64_t(first) * ld, range32(bytes));
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_readfirstlane(r[e]);
  return r;
}

__device__ __forceinline__ uint32_t lds_offset(const char* p) {
  return __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p))));
}

// 16 bytes' worth of fp32 sums to bf16.
__device__ __forceinline__ u32x4 pack_sums(const f32x4& x, const f32x4& y, float f) {
  return u32x4{pack_bf2(x[0] * f, x[1] * f), pack_bf2(x[2] * f, x[3] * f), pack_bf2(y[0] * f, y[1] * f), pack_bf2(y[2] * f, y[3] * f)};
}

// ---------------------------------------------------------------------------
// dq.  Wave (q, k) = (w % 2, w / 2) takes rows 64 q .. of the block and keys 32 k .. of each 64-key tile;
// the two waves of a row half meet in LDS at the end.
// A step interleaves, in a fixed order, the products dP(t) = V dO^T with the exponentials of S(t), then S(t + 1) =
// K Q^T with ds(t), then dQ^T += K^T dS^T(t): the matrix pipe does not wait for the vector units.
template <int DH>
__global__ __launch_bounds__(256, 1) void sparse_dq_bf16_kernel(const SparseArgs a) {
  constexpr int kC = DH / 16, kDT = DH / 32, kTB = kKB * DH * 2, kL = kTB / 4096, kBuf = 4;
  constexpr int kP = DH + 4;  // floats to a row of the sums
  constexpr int kBytes = std::max(2 * kBuf * kTB, 2 * 64 * kP * 4);
  __shared__ __attribute__((aligned(16))) char smem[kBytes];
  const int H = a.H, h = blockIdx.x % H, blk = blockIdx.x / H;
  const Seq s = seq_of<false>(a.seq, blk);
  const int lane = threadIdx.x % kWave, l32 = lane % 32, hi = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wq = wave % 2, wk = wave / 2;
  const int q_first = s.q_lo + (blk - s.qb) * kQB, q_end = std::min(s.q_hi, q_first + kQB);
  const bf16_t* K = static_cast<const bf16_t*>(a.k) + int64_t(h / a.group) * DH;
  const bf16_t* V = static_cast<const bf16_t*>(a.v) + int64_t(h / a.group) * DH;
  BlockWalk walk(a, h, blk, s.nk);
  const int n_tiles = walk.total;

  bf16x8 qf[2][kC], gf[2][kC];
  float lse2[2], delta[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = std::min(q_first + 64 * wq + 32 * t + l32, q_end - 1);
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + int64_t(row) * a.q_ld + h * DH + 8 * hi;
    const bf16_t* g = static_cast<const bf16_t*>(a.dout) + int64_t(row) * a.do_ld + h * DH + 8 * hi;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      qf[t][c] = as_bf16x8(*reinterpret_cast<const u32x4*>(q + 16 * c));
      gf[t][c] = as_bf16x8(*reinterpret_cast<const u32x4*>(g + 16 * c));
    }
    lse2[t] = a.lse[int64_t(h) * a.M + row] * kLog2e;
    delta[t] = a.delta[int64_t(h) * a.M + row];
  }
  f32x16 acc[2][kDT];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][dt][r] = 0.f;
  const float scale2 = kLog2e * a.scale;
  const Frag<DH> frag;
  uint32_t k_off[kL], v_off[kL];
#pragma unroll
  for (int i = 0; i < kL; ++i) {
    k_off[i] = load_off<DH>(wave + 4 * i, a.k_ld);
    v_off[i] = load_off<DH>(wave + 4 * i, a.v_ld);
  }
  const uint32_t lds_w = lds_offset(smem) + wave * 1024;
  auto load = [&](int buf, int j) {
    const int first = s.k_lo + j * kKB;
    const u32x4 rk = rows_rsrc(K, a.k_ld, first, s.k_hi, DH), rv = rows_rsrc(V, a.v_ld, first, s.k_hi, DH);
#pragma unroll
    for (int i = 0; i < kL; ++i) lds_load16(lds_w + 2 * buf * kTB, k_off[i], rk, 0, 4096 * i);
#pragma unroll
    for (int i = 0; i < kL; ++i) lds_load16(lds_w + (2 * buf + 1) * kTB, v_off[i], rv, 0, 4096 * i);
  };
  // Waits until at most `n` later tiles' loads are in flight.
  auto landed = [](int n) {
    if (n >= 2) vm_wait<4 * kL>();
    else if (n == 1) vm_wait<2 * kL>();
    else vm_wait<0>();
  };
  typedef f32x16 Pair[2];
  // Slots of a step: kC of dP, kC of S, 2 kDT of dQ, each a fragment and its two products.
  constexpr int kRd = 4, kSlots = 2 * kC + 2 * kDT;
  const char* half = smem + 32 * wk * (DH * 2);
  auto fragment = [&](int i, int buf, int nbuf) {
    if (i < kC) return frag.rows(half + (2 * buf + 1) * kTB, i);
    if (i < 2 * kC) return frag.rows(half + 2 * nbuf * kTB, i - kC);
    return frag.columns(half + 2 * buf * kTB, (i - 2 * kC) / kDT, (i - 2 * kC) % kDT);
  };
  // Keys past the last: no probability.
  auto mask = [&](int j, Pair& x) {
    const int up = s.k_hi - s.k_lo - j * kKB - 32 * wk;
    if (up >= 32) return;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r / 4) + r % 4 + 4 * hi >= up) x[0][r] = x[1][r] = -INFINITY;
  };
  // x: S(t), becoming probabilities; xn: S(t + 1).
  bf16x8 ds[2][2];
  auto step = [&](Pair& x, Pair& xn, int buf, int nbuf, auto before_s) {
    Pair dp = {};
    bf16x8 f[kRd];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kRd; ++i) f[i] = fragment(i, buf, nbuf);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      // The next tile's fragments may be read from here on.
      if (i + kRd == kC) before_s();
      const bf16x8 w = f[i % kRd];
      if (i < kC) {
        dp[0] = mfma32(w, gf[0][i], dp[0]);
        dp[1] = mfma32(w, gf[1][i], dp[1]);
      } else if (i < 2 * kC) {
        const int c = i - kC;
        xn[0] = mfma32(w, qf[0][c], c == 0 ? f32x16{} : xn[0]);
        xn[1] = mfma32(w, qf[1][c], c == 0 ? f32x16{} : xn[1]);
      } else {
        const int c = (i - 2 * kC) / kDT, dt = (i - 2 * kC) % kDT;
        acc[0][dt] = mfma32(w, ds[0][c], acc[0][dt]);
        acc[1][dt] = mfma32(w, ds[1][c], acc[1][dt]);
      }
      if (i + kRd < kSlots) f[i % kRd] = fragment(i + kRd, buf, nbuf);
      if (i < kC) {  // exponentials of 16 / kC registers of both
#pragma unroll
        for (int r = 16 * i / kC; r < 16 * (i + 1) / kC; ++r)
#pragma unroll
          for (int t = 0; t < 2; ++t) x[t][r] = __builtin_amdgcn_exp2f(fmaf(x[t][r], scale2, -lse2[t]));
      } else if (i < 2 * kC) {  // ds, packed in pairs
#pragma unroll
        for (int r = 16 * (i - kC) / kC; r < 16 * (i - kC + 1) / kC; ++r)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            x[t][r] *= dp[t][r] - delta[t];
            if (r % 2 == 1) put(ds[t][r / 8], r, x[t][r - 1], x[t][r]);
          }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  if (n_tiles > 0) {
    // Key blocks of tiles t and t + 1; loads run up to three tiles ahead.
    int j0 = walk.next(), j1 = -1, j2 = -1;
    load(0, j0);
    if (n_tiles > 1) load(1, j1 = walk.next());
    if (n_tiles > 2) load(2, j2 = walk.next());
    landed(n_tiles - 1);
    lds_barrier();
    Pair xa = {}, xb = {};
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const bf16x8 f = frag.rows(half, c);
      xa[0] = mfma32(f, qf[0][c], xa[0]);
      xa[1] = mfma32(f, qf[1][c], xa[1]);
    }
    auto one = [&](int t, Pair& x, Pair& xn) {
      mask(j0, x);
      step(x, xn, t & 3, (t + 1) & 3, [&]() {
        // Tile t + 1 has landed for every wave, and every wave is done with tile t - 1, whose place tile t + 3 takes.
        // (On the last tile what lies in the next place is read, and its products are not used.)
        if (t + 1 >= n_tiles) return;
        landed(std::min(1, n_tiles - t - 2));  // tile t + 2 may be on its way
        lds_barrier();
        j0 = j1;
        j1 = j2;
        if (t + 3 < n_tiles) load((t + 3) & 3, j2 = walk.next());
      });
    };
    int t = 0;
    for (; t + 1 < n_tiles; t += 2) {
      one(t, xa, xb);
      one(t + 1, xb, xa);
    }
    if (t < n_tiles) one(t, xa, xb);
  }
  // The two key halves: each wave leaves one 32-row half of its sums and adds the other's.
  lds_barrier();
  float* sums = reinterpret_cast<float*>(smem) + wq * 64 * kP;
  {
    const int give = 1 - wk;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& o = give ? acc[1][dt] : acc[0][dt];
        *reinterpret_cast<f32x4*>(sums + (32 * give + l32) * kP + 32 * dt + 8 * q + 4 * hi) =
            f32x4{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
      }
  }
  lds_barrier();
  const int row = q_first + 64 * wq + 32 * wk + l32;
  if (row >= q_end) return;
  bf16_t* dst = static_cast<bf16_t*>(a.dq) + int64_t(row) * a.dq_ld + h * DH + 4 * hi;
#pragma unroll
  for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x16& o = wk ? acc[1][dt] : acc[0][dt];
      f32x4 v = *reinterpret_cast<const f32x4*>(sums + (32 * wk + l32) * kP + 32 * dt + 8 * q + 4 * hi);
      // Key half 0 first, whichever wave adds.
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (o[4 * q + e] + v[e]) * a.scale;
      *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * q) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
    }
}

// ---------------------------------------------------------------------------
// dk and dv.  Wave w takes rows 32 w .. of every query block, all 64 keys, from LDS of its own: no
// barrier until the four waves' sums meet at the end.
constexpr int kItems = 4096;  // (head, query block) pairs looked at together

template <int DH>
__global__ __launch_bounds__(256, 1) void sparse_dkv_bf16_kernel(const SparseArgs a) {
  constexpr int kC = DH / 16, kDT = DH / 32, kTB = 32 * DH * 2, kL = kTB / 1024;
  constexpr int kP = DH + 4, kWaveBytes = 4 * kTB;  // two of the queries' and two of the gradients' tiles
  constexpr int kBytes = std::max(4 * kWaveBytes, 4 * 64 * kP * 4);
  __shared__ __attribute__((aligned(16))) char smem[kBytes];
  __shared__ __attribute__((aligned(16))) char vt[kKB * DH * 2];  // the key block's values
  __shared__ __attribute__((aligned(16))) float stats[4][64];
  __shared__ uint64_t bits[kItems / 64];
  const int Hk = a.H / a.group, hk = blockIdx.x % Hk, blk = blockIdx.x / Hk;
  const Seq s = seq_of<true>(a.seq, blk);
  const int lane = threadIdx.x % kWave, l32 = lane % 32, hi = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int k_first = s.k_lo + (blk - s.kb) * kKB, nq = (s.q_hi - s.q_lo + kQB - 1) / kQB, items = nq * a.group;

  // The keys stay in registers; for the values there is no room beside the sums (they spilled 89 registers).
  bf16x8 kf[2][kC];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = std::min(k_first + 32 * t + l32, s.k_hi - 1);  // keys past the last: not stored
    const bf16_t* k = static_cast<const bf16_t*>(a.k) + int64_t(row) * a.k_ld + hk * DH + 8 * hi;
#pragma unroll
    for (int c = 0; c < kC; ++c) kf[t][c] = as_bf16x8(*reinterpret_cast<const u32x4*>(k + 16 * c));
  }
  {
    const u32x4 rv = rows_rsrc(static_cast<const bf16_t*>(a.v) + int64_t(hk) * DH, a.v_ld, k_first, s.k_hi, DH);
#pragma unroll
    for (int i = 0; i < kKB * DH * 2 / 4096; ++i)
      lds_load16(lds_offset(vt) + wave * 1024, load_off<DH>(wave + 4 * i, a.v_ld), rv, 0, 4096 * i);
    vm_wait<0>();  // the barriers before the first step make it every wave's
  }
  f32x16 dk[2][kDT], dv[2][kDT];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[t][dt][r] = dv[t][dt][r] = 0.f;
  const float scale2 = kLog2e * a.scale, unscale = 1.f / a.scale;
  Frag<DH> frag;
  // An instruction's rows repeat their swizzle after kOff instructions.
  constexpr int kR = kWave / (DH / 8), kOff = 16 / kR, kRd = 4, kSlots = 2 * kC + 4 * kDT;
  static_assert(kSlots % kRd == 0, "the fragments' ring closes over a step");
  uint32_t q_off[kOff], g_off[kOff];
#pragma unroll
  for (int i = 0; i < kOff; ++i) {
    q_off[i] = load_off<DH>(i, a.q_ld);
    g_off[i] = load_off<DH>(i, a.do_ld);
  }
  char* mine = smem + wave * kWaveBytes;
  const uint32_t lds_w = lds_offset(mine);

  for (int base = 0; base < items; base += kItems) {
    const int n = std::min(kItems, items - base);
    __syncthreads();
    for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += 256) {
      const int e = base + i;
      const bool on = i < n && kept(a, hk * a.group + e / nq, s.qb + e % nq, blk - s.kb);
      const uint64_t w = __ballot(on);
      if (lane == 0) bits[i / 64] = w;
    }
    __syncthreads();
    // The kept pairs, one ahead of the products.
    int word = -1;
    uint64_t cur = 0;
    auto next = [&]() {
      while (cur == 0) {
        if (64 * ++word >= n) return -1;
        const uint64_t w = bits[word];
        cur = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(w >> 32)))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(w)));
      }
      const int i = 64 * word + __builtin_ctzll(cur);
      cur &= cur - 1;
      return base + i;
    };
    float stat = 0.f;  // lanes 0 .. 31: lse of the pair's rows that are on their way, the others: delta
    auto load = [&](int buf, int e) {
      const int h = hk * a.group + e / nq, first = s.q_lo + (e % nq) * kQB + 32 * wave;
      const u32x4 rq = rows_rsrc(static_cast<const bf16_t*>(a.q) + int64_t(h) * DH, a.q_ld, first, s.q_hi, DH);
      const u32x4 rg = rows_rsrc(static_cast<const bf16_t*>(a.dout) + int64_t(h) * DH, a.do_ld, first, s.q_hi, DH);
      const uint32_t q_step = uint32_t(a.q_ld) * (2 * kR), g_step = uint32_t(a.do_ld) * (2 * kR);
#pragma unroll
      for (int i = 0; i < kL; ++i) lds_load16(lds_w + 2 * buf * kTB, q_off[i % kOff], rq, i / kOff * kOff * q_step, 1024 * i);
#pragma unroll
      for (int i = 0; i < kL; ++i) lds_load16(lds_w + (2 * buf + 1) * kTB, g_off[i % kOff], rg, i / kOff * kOff * g_step, 1024 * i);
      // Rows past the last: no probability.
      const float* p = hi ? a.delta : a.lse;
      stat = hi ? 0.f : INFINITY;
      if (first + l32 < s.q_hi) stat = p[int64_t(h) * a.M + first + l32];
    };
    // A step's 32 (DH = 64: 16) slots, each a fragment and its two products, in a fixed order: S, dP with the
    // exponentials, dV with ds, dK with the start of the next step.
    f32x16 x[2], dp[2];
    bf16x8 f[kRd], vv[2][2], pb[2][2], db[2][2];
    auto fragment = [&](int i, const char* qt) {
      const char* gt = qt + kTB;
      if (i < kC) return frag.rows(qt, i);
      if (i < 2 * kC) return frag.rows(gt, i - kC);
      if (i < 2 * kC + 2 * kDT) return frag.columns(gt, (i - 2 * kC) / kDT, (i - 2 * kC) % kDT);
      return frag.columns(qt, (i - 2 * kC - 2 * kDT) / kDT, (i - 2 * kC - 2 * kDT) % kDT);
    };
    // The pair that has landed: logits less lse / scale, and dp less delta, start from what is taken away.
    auto begin = [&]() {
      vm_wait<0>();
      stats[wave][lane] = hi ? -stat : -stat * unscale;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 m = *reinterpret_cast<const f32x4*>(&stats[wave][8 * q + 4 * hi]);
        const f32x4 d = *reinterpret_cast<const f32x4*>(&stats[wave][32 + 8 * q + 4 * hi]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[0][4 * q + r] = x[1][4 * q + r] = m[r];
          dp[0][4 * q + r] = dp[1][4 * q + r] = d[r];
        }
      }
    };
    int e0 = next(), e1 = -1, buf = 0;
    if (e0 >= 0) {
      load(0, e0);
      begin();
      if ((e1 = next()) >= 0) load(1, e1);
#pragma unroll
      for (int i = 0; i < kRd; ++i) f[i] = fragment(i, mine);
    }
    while (e0 >= 0) {
      const char* qt = mine + 2 * buf * kTB;
      const char* nt = mine + 2 * (buf ^ 1) * kTB;
      frag.fresh();
#pragma unroll
      for (int i = 0; i < kSlots; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 w = f[i % kRd];
        if (i < kC) {
          x[0] = mfma32(w, kf[0][i], x[0]);
          x[1] = mfma32(w, kf[1][i], x[1]);
        } else if (i < 2 * kC) {
          dp[0] = mfma32(w, vv[i % 2][0], dp[0]);
          dp[1] = mfma32(w, vv[i % 2][1], dp[1]);
        } else if (i < 2 * kC + 2 * kDT) {
          const int c = (i - 2 * kC) / kDT, dt = (i - 2 * kC) % kDT;
          dv[0][dt] = mfma32(w, pb[0][c], dv[0][dt]);
          dv[1][dt] = mfma32(w, pb[1][c], dv[1][dt]);
        } else {
          const int c = (i - 2 * kC - 2 * kDT) / kDT, dt = (i - 2 * kC - 2 * kDT) % kDT;
          dk[0][dt] = mfma32(w, db[0][c], dk[0][dt]);
          dk[1][dt] = mfma32(w, db[1][c], dk[1][dt]);
        }
        if (i == 2 * kC + 2 * kDT && e1 >= 0) begin();
        if (i + 2 >= kC && i + 2 < 2 * kC) {
          vv[i % 2][0] = frag.rows(vt, i + 2 - kC);
          vv[i % 2][1] = frag.rows(vt + 32 * (DH * 2), i + 2 - kC);
        }
        // Near the end the next pair's first fragments (stale ones, unused, where there is none).
        f[i % kRd] = i + kRd < kSlots ? fragment(i + kRd, qt) : fragment(i + kRd - kSlots, nt);
        if (i >= kC && i < 2 * kC) {
#pragma unroll
          for (int r = 16 * (i - kC) / kC; r < 16 * (i - kC + 1) / kC; ++r)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              x[t][r] = __builtin_amdgcn_exp2f(x[t][r] * scale2);
              if (r % 2 == 1) put(pb[t][r / 8], r, x[t][r - 1], x[t][r]);
            }
        } else if (i >= 2 * kC && i < 2 * kC + 2 * kDT) {
          const int n = 2 * kDT, k = i - 2 * kC;
#pragma unroll
          for (int r = 16 * k / n; r < 16 * (k + 1) / n; ++r)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              dp[t][r] *= x[t][r];
              if (r % 2 == 1) put(db[t][r / 8], r, dp[t][r - 1], dp[t][r]);
            }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      // This pair's reads are done: its place is the one after the next's.
      e0 = e1;
      if (e0 >= 0) {
        asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(kRd) : "memory");
        if ((e1 = next()) >= 0) load(buf, e1);
      }
      buf ^= 1;
    }
  }
  // The waves' sums, dk's then dv's.
  float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& o = which ? dv[t][dt] : dk[t][dt];
          *reinterpret_cast<f32x4*>(sums + (64 * wave + 32 * t + l32) * kP + 32 * dt + 8 * q + 4 * hi) =
              f32x4{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
        }
    __syncthreads();
    bf16_t* out = static_cast<bf16_t*>(which ? a.dv : a.dk);
    const int64_t ld = which ? a.dv_ld : a.dk_ld;
    for (int i = threadIdx.x; i < 64 * (DH / 8); i += 256) {
      const int r = i / (DH / 8), c = i % (DH / 8) * 8;
      if (k_first + r >= s.k_hi) continue;
      f32x4 v[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float* p = sums + r * kP + c + 4 * u;
        f32x4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const f32x4*>(p + 64 * k * kP);
        v[u] = (w[0] + w[1]) + (w[2] + w[3]);
      }
      *reinterpret_cast<u32x4*>(out + int64_t(k_first + r) * ld + int64_t(hk) * DH + c) = pack_sums(v[0], v[1], which ? 1.f : a.scale);
    }
  }
}

template <int DH>
void launch_back(const SparseArgs& a, hipStream_t s) {
  const unsigned nq = unsigned(a.seq.q_blk[kMaxSeqs]), nk = unsigned(a.seq.k_blk[a.seq.B]);
  if (nq > 0) hipLaunchKernelGGL((sparse_dq_bf16_kernel<DH>), dim3(nq * unsigned(a.H)), dim3(256), 0, s, a);
  if (nk > 0) hipLaunchKernelGGL((sparse_dkv_bf16_kernel<DH>), dim3(nk * unsigned(a.H / a.group)), dim3(256), 0, s, a);
}

}  // namespace

void launch_sparse_back_bf16(const SparseArgs& a, hipStream_t s) {
  if (a.d == 128) launch_back<128>(a, s);
  else launch_back<64>(a, s);
}

}  // namespace avits
