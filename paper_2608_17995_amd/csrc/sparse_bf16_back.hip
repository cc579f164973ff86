// Backward pass of the attention over chosen key blocks in bf16, on v_mfma_f32_32x32x16_bf16.
//
// dq: a workgroup owns a query block of 128 rows of a head and walks the set bits of its mask row;
// dk, dv: a workgroup owns a key block of 64 rows and walks the query blocks of its key head's query
// heads that keep it.  Both make the logits and probabilities again from lse, so seven
// products run where five would do, and no sum crosses workgroups.
//
// Probabilities and ds are rounded to bf16 for the second products, which the matrix instruction
// takes; everything else is fp32.  For dq what the rounding of ds leaves over goes in as well, as a second operand: a row's
// ds add up to zero, so dq has nothing of what all keys have in common, but the roundings' errors do (with keys of which a
// third is shared by their neighbours, 110 rows: dq off by 0.0026 of its size, with the rest by 0.0017, its own rounding's;
// it costs 25 of 136 us at 4608 rows, 16 heads of 128, 30 % kept).  dk and dv are off by 0.0024.
// All this is against the formula with o as it is stored, in bf16.  What o lost reaches delta, and through it every ds of a row
// alike, so that dq takes it times the mean key: against the exact gradient of the inputs dq is off by 0.0017 where keys have little in
// common (110 rows and more, 4 heads), by 0.014 to 0.027 where they share eight times what they differ by.
#include <utility>

#include "sparse_plan.h"

namespace avits {
namespace {

// f(0), f(1), ... f(N - 1) with compile-time arguments.
template <int... I, class F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}
template <int N> using Int = std::integral_constant<int, N>;
#define AVITS_INLINE __attribute__((always_inline))

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

// Registers r - 1 and r (odd) of a product into their chunk of the next product's operand; the pair as it was rounded.
__device__ __forceinline__ uint32_t put(bf16x8& chunk, int r, float lo, float up) {
  u32x4 v = __builtin_bit_cast(u32x4, chunk);
  v[(r % 8) / 2] = pack_bf2(lo, up);
  chunk = as_bf16x8(v);
  return v[(r % 8) / 2];
}

// A wave's share of a tile of ROWS rows that four (64 rows) or eight waves load: instructions of 1 KB, whose
// lanes fill LDS in order, so the swizzle is in where each lane reads.
template <int DH, int ROWS, int NW = ROWS == 128 ? 8 : 4>
struct TileLoad {
  static constexpr int kCH = DH / 8, kR = kWave / kCH, kN = ROWS * DH * 2 / 1024 / NW;
  uint32_t row, chunk;  // the first instruction's row and swizzled chunk, in bytes
  int64_t ld2;          // bytes to a row
  __device__ __forceinline__ TileLoad(int64_t ld, int wave) : ld2(ld * 2) {
    const int lane = threadIdx.x % kWave, r = kR * kN * wave + lane / kCH;
    row = uint32_t(r) * uint32_t(ld * 2);
    chunk = uint32_t(((lane % kCH) ^ swz<DH>(r)) * 16);
  }
  // Instruction i is kR i rows on, where the swizzle differs in bits of i (rows kR kN wave are even enough).
  __device__ __forceinline__ uint32_t off(int i) const {
    return row + (chunk ^ uint32_t((DH == 128 ? 16 : 32) * i)) + i * (kR * uint32_t(ld2));
  }
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row), "+v"(chunk)); }
  // Rows first .. of a head, those from `end` on as zeros.  (A tile that starts past the last row is not asked for.)
  __device__ __forceinline__ u32x4 rows(const bf16_t* base, int first, int end) const {
    return at(reinterpret_cast<const char*>(base) + first * ld2, int64_t(end - first - 1) * ld2 + DH * 2);
  }
  __device__ __forceinline__ static u32x4 at(const char* p, int64_t bytes) {
    u32x4 r = buffer_rsrc(p, bytes >> 32 ? 0xffffffffu : uint32_t(bytes));
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_readfirstlane(r[e]);
    return r;
  }
  // Load i of them, to LDS byte dst + 1024 i.
  __device__ __forceinline__ void one(int i, const u32x4& r, uint32_t dst) const {
    lds_load16(dst, off(i), r, 0, 1024 * i);
  }
  __device__ __forceinline__ void all(const u32x4& r, uint32_t dst) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) one(i, r, dst);
  }
};

__device__ __forceinline__ uint32_t lds_offset(const char* p) {
  return __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p))));
}

// The lane's sums of one row (register r of tile dt: column 32 dt + 8 (r / 4) + 4 (l / 32) + r % 4), times f.
template <int DH>
__device__ __forceinline__ void store_sums(bf16_t* dst, const f32x16* o, float f) {
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * q) =
          u32x2{pack_bf2(o[dt][4 * q] * f, o[dt][4 * q + 1] * f), pack_bf2(o[dt][4 * q + 2] * f, o[dt][4 * q + 3] * f)};
}

// ---------------------------------------------------------------------------
// dq: 32 rows to a wave.  A step takes a 64-key tile in two halves of 32 keys; the exponentials of one run
// under the products of the other, and under the other wave's of the SIMD.  4608 rows, 16 heads of 128, text and 14 of 64
// blocks kept: 132 us, 1.0 PFLOP/s of the four products that it makes (64 rows to a wave 148, with three of them).
template <int DH>
__global__ __launch_bounds__(256, 2) void sparse_dq_bf16_kernel(const SparseArgs a) {
  constexpr int kC = DH / 16, kDT = DH / 32, kTB = kKB * DH * 2, kL = kTB / 4096;
  __shared__ __attribute__((aligned(16))) char smem[4 * kTB];
  const int H = a.H, units = a.seq.q_blk[kMaxSeqs] * H;
  const int4 item = sparse_item(a, units, blockIdx.x);
  if (item.x < 0) return;
  const int h = item.x % H, blk = item.x / H, piece = item.y & 0xffff, pieces = item.y >> 16;
  const Seq s = seq_of<false>(a.seq, blk);
  const int lane = threadIdx.x % kWave, l32 = lane % 32, hi = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int q_first = s.q_lo + (blk - s.qb) * kQB, q_end = std::min(s.q_hi, q_first + kQB);
  const bf16_t* K = static_cast<const bf16_t*>(a.k) + int64_t(h / a.group) * DH;
  const bf16_t* V = static_cast<const bf16_t*>(a.v) + int64_t(h / a.group) * DH;
  BlockWalk walk(a, h, blk, s.nk);
  const int t_lo = int(int64_t(walk.total) * piece / pieces), n_tiles = int(int64_t(walk.total) * (piece + 1) / pieces) - t_lo;
  const int row = q_first + 32 * wave + l32;
  walk.skip(t_lo);

  bf16x8 qf[kC], gf[kC];
  f32x16 acc[kDT];
  const int from = std::min(row, q_end - 1);
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q) + int64_t(from) * a.q_ld + h * DH + 8 * hi;
    const bf16_t* g = static_cast<const bf16_t*>(a.dout) + int64_t(from) * a.do_ld + h * DH + 8 * hi;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      qf[c] = as_bf16x8(*reinterpret_cast<const u32x4*>(q + 16 * c));
      gf[c] = as_bf16x8(*reinterpret_cast<const u32x4*>(g + 16 * c));
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
  }
  const float2 st = a.stats[int64_t(h) * a.M + from];
  const float lse2 = st.x * kLog2e, delta = st.y;
  const float scale2 = kLog2e * a.scale;
  Frag<DH> frag;
  TileLoad<DH, kKB> lk(a.k_ld, wave), lv(a.v_ld, wave);
  const uint32_t lds_w = lds_offset(smem) + wave * (kL * 1024);
  // The next tile's buffers; its loads are spread over a step's first products: issued together they hold
  // up the wave, and the products behind them, until the CU has taken them (1 KB in 16 cycles).
  u32x4 rk, rv;
  auto next_tile = [&](int j) {
    rk = lk.rows(K, s.k_lo + j * kKB, s.k_hi);
    rv = lv.rows(V, s.k_lo + j * kKB, s.k_hi);
  };
  // Slots of a step, each a fragment and its product: S and dP of half 0, of half 1, dQ of half 0, of half 1.
  constexpr int kRd = 4, kG = 2 * kC, kQ = 2 * kDT, kSlots = 2 * kG + 2 * kQ;
  f32x16 x[2], dp[2];
  bf16x8 ds[2][2], rest[2][2];
  // Of half t: probabilities and ds, element n of 16.
  auto grad = [&](auto tt, auto nn) AVITS_INLINE {
    constexpr int t = decltype(tt)::value, n = decltype(nn)::value;
    x[t][n] = __builtin_amdgcn_exp2f(fmaf(x[t][n], scale2, -lse2)) * (dp[t][n] - delta);
    if constexpr (n % 2 == 1) {
      const uint32_t pair = put(ds[t][n / 8], n, x[t][n - 1], x[t][n]);
      put(rest[t][n / 8], n, x[t][n - 1] - __uint_as_float(pair << 16), x[t][n] - __uint_as_float(pair & 0xffff0000u));
    }
  };
  if (n_tiles > 0) {
    int j0 = walk.next(), buf = 0;
    next_tile(j0);
    lk.all(rk, lds_w);
    lv.all(rv, lds_w + kTB);
    for (int t = 0; t < n_tiles; ++t) {
      // This tile has landed for every wave, and every wave is done with the last, whose place the next takes.
      vm_wait<0>();
      lds_barrier();
      const int j = j0;
      const bool more = t + 1 < n_tiles;
      const uint32_t next_at = lds_w + 2 * (buf ^ 1) * kTB;
      const char* kt = smem + 2 * buf * kTB;
      const char* vt = kt + kTB;
      const int up = s.k_hi - s.k_lo - j * kKB - 4 * hi;
      frag.fresh();
      auto fragment = [&](auto ii) AVITS_INLINE {
        constexpr int i = decltype(ii)::value;
        if constexpr (i < 2 * kG) {
          constexpr int half = i / kG, c = i % kG;
          return frag.rows((c < kC ? kt : vt) + 32 * half * (DH * 2), c % kC);
        } else {
          constexpr int k = i - 2 * kG;
          return frag.columns(kt, k / kDT, k % kDT);
        }
      };
      bf16x8 f[kRd];
      __builtin_amdgcn_sched_barrier(0);
      each<kRd>([&](auto i) AVITS_INLINE { f[decltype(i)::value] = fragment(i); });
      each<kSlots>([&](auto slot) AVITS_INLINE {
        constexpr int i = decltype(slot)::value;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (i == kG || i == 2 * kG) {
          // Keys past the last: no probability.
          constexpr int half = i / kG - 1;
          if (up - 32 * half < 32 - 4 * hi) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (32 * half + 8 * (r / 4) + r % 4 >= up) x[half][r] = -INFINITY;
          }
        }
        if constexpr (i < 2 * kG) {
          constexpr int half = i / kG, c = i % kG;
          if constexpr (c < kC) x[half] = mfma32(f[i % kRd], qf[c], c == 0 ? f32x16{} : x[half]);
          else dp[half] = mfma32(f[i % kRd], gf[c - kC], c == kC ? f32x16{} : dp[half]);
        } else {
          constexpr int k = i - 2 * kG, c = k / kDT;
          acc[k % kDT] = mfma32(f[i % kRd], ds[c / 2][c % 2], acc[k % kDT]);
          acc[k % kDT] = mfma32(f[i % kRd], rest[c / 2][c % 2], acc[k % kDT]);
        }
        if constexpr (i + kRd < kSlots) f[i % kRd] = fragment(Int<i + kRd>{});
        if constexpr (i == 1)
          if (more) next_tile(j0 = walk.next());
        if constexpr (i >= 3 && i % 2 == 1 && i / 2 - 1 < 2 * kL) {
          constexpr int k = i / 2 - 1;
          if (more) k < kL ? lk.one(k, rk, next_at) : lv.one(k - kL, rv, next_at + kTB);
        }
        if constexpr (i >= kG && i < 2 * kG) {
          constexpr int n = i - kG;
          each<16 * (n + 1) / kG - 16 * n / kG>([&](auto e) AVITS_INLINE { grad(Int<0>{}, Int<16 * n / kG + decltype(e)::value>{}); });
        } else if constexpr (i >= 2 * kG && i < 2 * kG + kQ) {
          constexpr int n = i - 2 * kG;
          each<16 * (n + 1) / kQ - 16 * n / kQ>([&](auto e) AVITS_INLINE { grad(Int<1>{}, Int<16 * n / kQ + decltype(e)::value>{}); });
        }
      });
      __builtin_amdgcn_sched_barrier(0);
      buf ^= 1;
    }
  }
  if (row >= q_end) return;
  if (pieces > 1) {  // a piece: its sums to its slot
    float* to = a.part + (sparse_slot(a, units, item.w, piece) * kQB + (row - q_first)) * DH + 4 * hi;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(to + 32 * dt + 8 * q) =
            f32x4{acc[dt][4 * q], acc[dt][4 * q + 1], acc[dt][4 * q + 2], acc[dt][4 * q + 3]};
    return;
  }
  bf16_t* dst = static_cast<bf16_t*>(a.dq) + int64_t(row) * a.dq_ld + h * DH + 4 * hi;
  store_sums<DH>(dst, acc, grad_scale(a, s));
}

// ---------------------------------------------------------------------------
// dk and dv.  Eight waves: wave (k, q) = (w % 2, w / 2) takes keys 32 k .. and rows 32 q .. of each query block; the
// four waves of a key half meet in LDS at the end.
// The values' fragments stay in registers, the keys' are read from LDS: with both in registers no more
// than two fragments could be under way, and every product waited for its own (200 us at 4608
// rows, 16 heads of 128, text and 14 of 64 blocks kept; this takes 180 to 200).  Of 4900 cycles a step the matrix instructions
// take 2048 and LDS 1740; a workgroup's beginning and end take 7.7 us, and a CU has four or five.
constexpr int kItems = 1024;  // (head, query block) pairs looked at together

template <int DH>
__global__ __launch_bounds__(512, 2) void sparse_dkv_bf16_kernel(const SparseArgs a) {
  constexpr int kC = DH / 16, kDT = DH / 32, kTB = kQB * DH * 2;
  constexpr int kP = DH + 4;  // floats to a row of the sums
  constexpr int kBytes = std::max(4 * kTB, 8 * 32 * kP * 4);
  __shared__ __attribute__((aligned(16))) char smem[kBytes];
  __shared__ __attribute__((aligned(16))) char keys[kKB * DH * 2];
  __shared__ __attribute__((aligned(16))) float stats[8][64];
  __shared__ uint64_t bits[kItems / 64];
  __shared__ __attribute__((aligned(8))) int2 list[kItems];  // kept pairs: first row less the sequence's, head of the group
  const int Hk = a.H / a.group, units = a.seq.k_blk[kMaxSeqs] * Hk;
  const int4 item = sparse_item(a, units, blockIdx.x);
  if (item.x < 0) return;
  const int hk = item.x % Hk, blk = item.x / Hk, piece = item.y & 0xffff, pieces = item.y >> 16;
  const Seq s = seq_of<true>(a.seq, blk);
  const int lane = threadIdx.x % kWave, l32 = lane % 32, hi = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wk = wave % 2, wq = wave / 2;
  const int k_first = s.k_lo + (blk - s.kb) * kKB, nq = (s.q_hi - s.q_lo + kQB - 1) / kQB, items = nq * a.group;
  const int row = k_first + 32 * wk + l32;

  bf16x8 vf[kC];
  {
    const int from = std::min(row, s.k_hi - 1);  // keys past the last: not stored
    const bf16_t* v = static_cast<const bf16_t*>(a.v) + int64_t(from) * a.v_ld + hk * DH + 8 * hi;
#pragma unroll
    for (int c = 0; c < kC; ++c) vf[c] = as_bf16x8(*reinterpret_cast<const u32x4*>(v + 16 * c));
  }
  f32x16 dk[kDT], dv[kDT];
#pragma unroll
  for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[dt][r] = dv[dt][r] = 0.f;
  const float scale2 = kLog2e * a.scale, unscale = 1.f / a.scale;
  Frag<DH> frag;
  TileLoad<DH, kQB> lq(a.q_ld, wave), lg(a.do_ld, wave);
  constexpr int kShare = kTB / 8;  // bytes of a tile that a wave loads
  const uint32_t lds_w = lds_offset(smem) + wave * kShare;
  {
    const TileLoad<DH, kKB, 8> lk(a.k_ld, wave);
    lk.all(lk.rows(static_cast<const bf16_t*>(a.k) + int64_t(hk) * DH, k_first, s.k_hi), lds_offset(keys) + wave * (kKB * DH * 2 / 8));
  }

  // Pairs before this piece's, and its own.
  int skip = int(int64_t(item.z) * piece / pieces), left = pieces > 1 ? int(int64_t(item.z) * (piece + 1) / pieces) - skip : 0x7fffffff;
  const int64_t q_bytes = int64_t(s.q_hi - s.q_lo - 1) * lq.ld2 + DH * 2, g_bytes = int64_t(s.q_hi - s.q_lo - 1) * lg.ld2 + DH * 2;
  const char* Q = static_cast<const char*>(a.q) + int64_t(s.q_lo) * lq.ld2 + int64_t(hk) * a.group * (DH * 2);
  const char* G = static_cast<const char*>(a.dout) + int64_t(s.q_lo) * lg.ld2 + int64_t(hk) * a.group * (DH * 2);
  const float2* stats_of = a.stats + int64_t(hk) * a.group * a.M + s.q_lo;
  for (int base = 0; base < items; base += kItems) {
    const int n = std::min(kItems, items - base);
    __syncthreads();
    for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += 512) {
      const int e = base + i;
      const bool on = i < n && kept(a, hk * a.group + e / nq, s.qb + e % nq, blk - s.kb);
      const uint64_t w = __ballot(on);
      if (lane == 0) bits[i / 64] = w;
    }
    __syncthreads();
    int found = 0;  // the kept pairs, in order
    for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += 512) {
      const int e = base + i;
      int before = 0;
      for (int w = 0; w < i / 64; ++w) before += __popcll(bits[w]);
      const uint64_t w = bits[i / 64];
      if (w >> lane & 1) list[before + __popcll(w & ((uint64_t(1) << lane) - 1))] = make_int2(e % nq * kQB, e / nq);
    }
    for (int w = 0; 64 * w < n; ++w) found += __popcll(bits[w]);
    found = __builtin_amdgcn_readfirstlane(found);
    __syncthreads();
    int at = std::min(skip, found);
    const int end = int(std::min<int64_t>(found, int64_t(at) + left));
    skip -= at;
    left -= end - at;
    int h1 = 0, row1 = 0;  // the pair whose rows come next
    auto read = [&](int k) {
      const int2 e = list[k];
      row1 = __builtin_amdgcn_readfirstlane(e.x);
      h1 = __builtin_amdgcn_readfirstlane(e.y);
    };
    float stat = 0.f;  // lanes 0 .. 31: lse of the wave's rows of the tile on its way, the others: delta
    // The next pair's buffers; its loads are spread over a step's first products: issued together they hold
    // up the wave, and the products behind them, until the CU has taken them (1 KB in 16 cycles).
    u32x4 rq, rg;
    constexpr int kN = TileLoad<DH, kQB>::kN;
    auto next_pair = [&]() AVITS_INLINE {
      const int64_t qo = row1 * lq.ld2, go = row1 * lg.ld2;
      rq = lq.at(Q + qo + h1 * (DH * 2), q_bytes - qo);
      rg = lg.at(G + go + h1 * (DH * 2), g_bytes - go);
      // Rows past the last: no probability.
      const int r = row1 + 32 * wq + l32;
      stat = hi ? 0.f : INFINITY;
      const float* st = reinterpret_cast<const float*>(stats_of + int64_t(h1) * a.M + row1);
      if (r < s.q_hi - s.q_lo) stat = st[uint32_t(2 * (32 * wq + l32) + hi)];
    };
    // Slots of a step, each a fragment and its product: S (with a fragment of the keys too), dP, dV, dK.
    constexpr int kRd = 4, kRk = 3, kQ = 2 * kDT, kSlots = 2 * kC + 2 * kQ;
    int buf = 0;
    if (at < end) {
      read(at);
      next_pair();
      lq.all(rq, lds_w);
      lg.all(rg, lds_w + kTB);
    }
    for (; at < end; ++at) {
      // The tile has landed for every wave, and every wave is done with the last, whose place the next takes.
      vm_wait<0>();
      stats[wave][lane] = hi ? -stat : -stat * unscale;
      const bool more = at + 1 < end;
      if (more) read(at + 1);
      lds_barrier();
      const uint32_t next_at = lds_w + 2 * (buf ^ 1) * kTB;
      const char* qt = smem + 2 * buf * kTB + 32 * wq * (DH * 2);
      const char* gt = qt + kTB;
      const char* kt = keys + 32 * wk * (DH * 2);
      f32x16 x, dp;
      bf16x8 f[kRd], fk[kRk], pb[2], db[2];
      frag.fresh();
      lq.fresh();
      lg.fresh();
      auto fragment = [&](auto ii) AVITS_INLINE {
        constexpr int i = decltype(ii)::value;
        if constexpr (i < kC) return frag.rows(qt, i);
        else if constexpr (i < 2 * kC) return frag.rows(gt, i - kC);
        else if constexpr (i < 2 * kC + kQ) return frag.columns(gt, (i - 2 * kC) / kDT, (i - 2 * kC) % kDT);
        else return frag.columns(qt, (i - 2 * kC - kQ) / kDT, (i - 2 * kC - kQ) % kDT);
      };
      // Logits less lse / scale, and dp less delta, start from what is taken away.
      auto begin = [&](f32x16& y, int at) AVITS_INLINE {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 m = *reinterpret_cast<const f32x4*>(&stats[wave][at + 8 * q + 4 * hi]);
#pragma unroll
          for (int r = 0; r < 4; ++r) y[4 * q + r] = m[r];
        }
      };
      begin(x, 0);
      __builtin_amdgcn_sched_barrier(0);
      each<kRk>([&](auto i) AVITS_INLINE { fk[decltype(i)::value] = frag.rows(kt, decltype(i)::value); });
      each<kRd>([&](auto i) AVITS_INLINE { f[decltype(i)::value] = fragment(i); });
      each<kSlots>([&](auto slot) AVITS_INLINE {
        constexpr int i = decltype(slot)::value;
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 w = f[i % kRd];
        if constexpr (i < kC) x = mfma32(w, fk[i % kRk], x);
        else if constexpr (i < 2 * kC) dp = mfma32(w, vf[i - kC], dp);
        else if constexpr (i < 2 * kC + kQ) dv[(i - 2 * kC) % kDT] = mfma32(w, pb[(i - 2 * kC) / kDT], dv[(i - 2 * kC) % kDT]);
        else dk[(i - 2 * kC - kQ) % kDT] = mfma32(w, db[(i - 2 * kC - kQ) / kDT], dk[(i - 2 * kC - kQ) % kDT]);
        if constexpr (i + kRk < kC) fk[i % kRk] = frag.rows(kt, i + kRk);
        if constexpr (i == kC - kRk) begin(dp, 32);
        if constexpr (i + kRd < kSlots) f[i % kRd] = fragment(Int<i + kRd>{});
        if constexpr (i == 1)
          if (more) next_pair();
        if constexpr (i >= 3 && i % 2 == 1 && i / 2 - 1 < 2 * kN) {
          constexpr int k = i / 2 - 1;
          if (more) k < kN ? lq.one(k, rq, next_at) : lg.one(k - kN, rg, next_at + kTB);
        }
        if constexpr (i >= kC && i < 2 * kC) {  // exponentials under dP
          constexpr int k = i - kC;
          each<16 * (k + 1) / kC - 16 * k / kC>([&](auto e) AVITS_INLINE {
            constexpr int r = 16 * k / kC + decltype(e)::value;
            x[r] = __builtin_amdgcn_exp2f(x[r] * scale2);
            if constexpr (r % 2 == 1) put(pb[r / 8], r, x[r - 1], x[r]);
          });
        } else if constexpr (i >= 2 * kC && i < 2 * kC + kQ) {  // ds under dV
          constexpr int k = i - 2 * kC;
          each<16 * (k + 1) / kQ - 16 * k / kQ>([&](auto e) AVITS_INLINE {
            constexpr int r = 16 * k / kQ + decltype(e)::value;
            dp[r] *= x[r];
            if constexpr (r % 2 == 1) put(db[r / 8], r, dp[r - 1], dp[r]);
          });
        }
      });
      __builtin_amdgcn_sched_barrier(0);
      buf ^= 1;
    }
  }
  // The four row quarters p of a key half, as (p0 + p2) + (p1 + p3): quarters 0 and 1 take dk and give dv, 2 and 3 the
  // other way round; then quarter 1 gives its dk to 0, and 3 its dv to 2.
  vm_wait<0>();  // the keys, where no pair was kept
  float* sums = reinterpret_cast<float*>(smem);
  auto give = [&](const f32x16* o) {
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(sums + (32 * wave + l32) * kP + 32 * dt + 8 * q + 4 * hi) =
            f32x4{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
  };
  auto take = [&](f32x16* o, int from, bool first) {  // first: the other's sum stands first
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(sums + (32 * from + l32) * kP + 32 * dt + 8 * q + 4 * hi);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[dt][4 * q + r] = first ? v[r] + o[dt][4 * q + r] : o[dt][4 * q + r] + v[r];
      }
  };
  __syncthreads();
  if (wq < 2) give(dv);
  else give(dk);
  __syncthreads();
  if (wq < 2) take(dk, wave + 4, false);
  else take(dv, wave - 4, true);
  __syncthreads();
  if (wq == 1) give(dk);
  if (wq == 3) give(dv);
  __syncthreads();
  if (wq % 2 == 1) return;
  if (wq == 0) take(dk, wave + 2, false);
  else take(dv, wave + 2, false);
  if (row >= s.k_hi) return;
  if (pieces > 1) {
    float* slot = a.part + ((sparse_slot(a, units, item.w, piece) * 2 + (wq == 2)) * kKB + 32 * wk + l32) * DH + 4 * hi;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& o = wq == 2 ? dv[dt] : dk[dt];
        *reinterpret_cast<f32x4*>(slot + 32 * dt + 8 * q) = f32x4{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
      }
    return;
  }
  if (wq == 2) store_sums<DH>(static_cast<bf16_t*>(a.dv) + int64_t(row) * a.dv_ld + int64_t(hk) * DH + 4 * hi, dv, 1.f);
  else store_sums<DH>(static_cast<bf16_t*>(a.dk) + int64_t(row) * a.dk_ld + int64_t(hk) * DH + 4 * hi, dk, grad_scale(a, s));
}

// The pieces of cut lists added up in order: eight columns to a thread.  dq: 128 rows to a unit; dk, dv: 64 of each.  5 us
// for dq of 4608 rows of 16 heads of 128.
template <int DH, bool KEYS>
__global__ __launch_bounds__(256) void sparse_sum_kernel(const SparseArgs a) {
  constexpr int kL = DH / 8, kR = 256 / kL, kPer = kQB / kR;
  const int4 cut = sparse_cut(a, blockIdx.x / kPer);
  if (cut.x < 0) return;
  const int Hu = KEYS ? a.H / a.group : a.H;
  const int blk = cut.x / Hu, h = cut.x % Hu, r = blockIdx.x % kPer * kR + threadIdx.x / kL, c = threadIdx.x % kL * 8;
  const Seq s = seq_of<KEYS>(a.seq, blk);
  const bool is_dv = KEYS && r >= kKB;
  const int row = KEYS ? s.k_lo + (blk - s.kb) * kKB + r % kKB : s.q_lo + (blk - s.qb) * kQB + r;
  if (row >= (KEYS ? s.k_hi : s.q_hi)) return;
  const float* p = a.part + (cut.z * int64_t(kQB) + r) * DH + c;
  constexpr int64_t step = int64_t(kQB) * DH;  // a plan's pieces (no lists are cut without one here) have consecutive slots
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll 4
  for (int i = 0; i < cut.y; ++i) {
    x += *reinterpret_cast<const f32x4*>(p + i * step);
    y += *reinterpret_cast<const f32x4*>(p + i * step + 4);
  }
  const float f = is_dv ? 1.f : grad_scale(a, s);
  x *= f, y *= f;
  bf16_t* out = static_cast<bf16_t*>(KEYS ? (is_dv ? a.dv : a.dk) : a.dq);
  const int64_t ld = KEYS ? (is_dv ? a.dv_ld : a.dk_ld) : a.dq_ld;
  *reinterpret_cast<u32x4*>(out + int64_t(row) * ld + int64_t(h) * DH + c) =
      u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
}

template <int DH>
void launch_back(const SparseArgs& q, const SparseArgs& k, hipStream_t s) {
  constexpr int kPer = kQB * DH / 8 / 256;
  const int64_t uq = int64_t(q.seq.q_blk[kMaxSeqs]) * q.H, uk = int64_t(q.seq.k_blk[kMaxSeqs]) * (q.H / q.group);
  if (uq > 0) hipLaunchKernelGGL((sparse_dq_bf16_kernel<DH>), dim3(unsigned(uq + q.slots)), dim3(256), 0, s, q);
  if (uk > 0) hipLaunchKernelGGL((sparse_dkv_bf16_kernel<DH>), dim3(unsigned(uk + k.slots)), dim3(512), 0, s, k);
  if (q.plan) hipLaunchKernelGGL((sparse_sum_kernel<DH, false>), dim3(unsigned(std::min<int64_t>(kShares, q.slots) * kPer)), dim3(256), 0, s, q);
  if (k.plan) hipLaunchKernelGGL((sparse_sum_kernel<DH, true>), dim3(unsigned(std::min<int64_t>(kShares, k.slots) * kPer)), dim3(256), 0, s, k);
}

}  // namespace

void launch_sparse_back_bf16(const SparseArgs& q, const SparseArgs& k, hipStream_t s) {
  if (q.d == 128) launch_back<128>(q, k, s);
  else launch_back<64>(q, k, s);
}

}  // namespace avits
