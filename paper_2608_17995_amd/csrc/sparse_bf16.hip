// Attention over chosen key blocks in bf16, forward.
//
// One 256-thread workgroup per (query block of 128 rows, head), 32 rows to a wave, two
// workgroups per CU; it walks the set bits of its mask row.  Key and value tiles of
// 64 rows go from memory to LDS directly, two of each in flight or in use.  The
// products of a step (P(t - 1) V and S(t + 1) = K Q^T) do not depend on its softmax (of S(t)),
// so a wave issues them interleaved, in a fixed order.
// Both products run on v_mfma_f32_32x32x16_bf16 in transposed form:
//   S^T = K Q^T   -> lane l holds query row l % 32; register r of a 32-key sub-tile is key
//                    8 (r / 4) + 4 (l / 32) + r % 4,
//   O^T = V^T P^T -> the lane's 16 head-dim values of the same row.
// So the probabilities are, register for register, the second product's operand, if its other
// operand holds V's keys in that order: four keys at a time of one column, which is what
// ds_read_b64_tr_b16 makes of four rows of V as they lie in memory.
// Probabilities are rounded to bf16 for the product with V, which the matrix
// instruction takes; maxima, sums and outputs are fp32.  An exponent is fma(s, scale log2 e, -maximum), whose product is exact but whose
// maximum was rounded: all of a row's probabilities carry 2 to the power of that rounding, which their sum takes away
// again.  From logits of 2^31 on it could leave fp32.
//
// Bound by the matrix instructions and, at heads of 64, the exponentials: 16896 rows of 16 heads of 128, a quarter kept, 600 us,
// 1.04 PFLOP/s (a large library product 1.2); 5171 rows of 16 heads of 64, 40 us, 0.52 (three workgroups
// to a CU the same).
//
// Long lists are cut into pieces (by a plan, or all alike where there are few units), whose
// unnormalised outputs and (max, sum) a second kernel joins in key order.
#include <type_traits>

#include "sparse_plan.h"

namespace avits {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNone = -3e38f;  // a running maximum below every logit

template <int DH>
__global__ __launch_bounds__(256, 2) void sparse_bf16_kernel(const SparseArgs a) {
  constexpr int NW = 4;                    // waves
  constexpr int kKT = 64;                  // keys to a tile
  constexpr int kC = DH / 16;              // k steps of S
  constexpr int kDT = DH / 32;             // 32-row tiles of O^T
  constexpr int kCH = DH / 8;              // 16-byte chunks of a row
  constexpr int kRows = kWave / kCH;       // rows to a load instruction
  constexpr int kTB = kKT * DH * 2;        // bytes of a tile
  constexpr int kL = kTB / 1024 / NW;      // load instructions to a wave and tile
  // Two K tiles, then two V tiles, unpadded: chunk c of row r lies at c ^ swz_k(r) (K) or c ^ swz(r) (V), so that the fragment
  // reads (16 rows of one chunk; four rows of four chunks) touch every bank once.
  __shared__ __attribute__((aligned(16))) char smem[4 * kTB];

  const int H = a.H, units = a.seq.q_blk[kMaxSeqs] * H;
  const int4 item = sparse_item(a, units, blockIdx.x);
  if (item.x < 0) return;
  const int h = item.x % H, blk = item.x / H, piece = item.y & 0xffff, pieces = item.y >> 16;
  const Seq s = seq_of<false>(a.seq, blk);
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int l32 = lane % 32, hi = lane / 32;
  const int q_first = s.q_lo + (blk - s.qb) * kQB, q_end = std::min(s.q_hi, q_first + kQB);
  const int row = q_first + wave * 32 + l32;

  BlockWalk walk(a, h, blk, s.nk);
  const int t_lo = int(int64_t(walk.total) * piece / pieces), t_hi = int(int64_t(walk.total) * (piece + 1) / pieces);
  const int n_tiles = t_hi - t_lo;
  walk.skip(t_lo);

  float mrow = kNone, lrow = 0.f;
  f32x16 oacc[kDT];
#pragma unroll
  for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;

  if (n_tiles > 0) {
    const bf16_t* K = static_cast<const bf16_t*>(a.k) + int64_t(h / a.group) * DH;
    const bf16_t* V = static_cast<const bf16_t*>(a.v) + int64_t(h / a.group) * DH;
    bf16x8 qf[kC];
    {
      const bf16_t* src = static_cast<const bf16_t*>(a.q) + int64_t(std::min(row, q_end - 1)) * a.q_ld + h * DH + 8 * hi;
#pragma unroll
      for (int c = 0; c < kC; ++c) qf[c] = as_bf16x8(*reinterpret_cast<const u32x4*>(src + 16 * c));
    }
    const float scale2 = kLog2e * a.scale;
    auto swz_k = [](int r) { return DH == 128 ? r & 15 : (r >> 1) & 7; };
    uint32_t k_off[kL], v_off[kL];
#pragma unroll
    for (int j = 0; j < kL; ++j) {
      const int r = kRows * (wave + NW * j) + lane / kCH;
      k_off[j] = uint32_t(r) * uint32_t(a.k_ld * 2) + uint32_t(((lane % kCH) ^ swz_k(r)) * 16);
      v_off[j] = uint32_t(r) * uint32_t(a.v_ld * 2) + uint32_t(((lane % kCH) ^ swz<DH>(r)) * 16);
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(
        uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(&smem[0]))));
    const uint32_t lds_w = lds0 + wave * 1024;
    auto uniform = [](u32x4 r) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_readfirstlane(r[e]);
      return r;
    };
    // Rows past the sequence's last come back as zeros.
    auto rows_of = [&](const bf16_t* base, int64_t ld, int j) {
      const int first = s.k_lo + j * kKB;
      const int64_t bytes = (int64_t(s.k_hi - first - 1) * ld + DH) * 2;
      return uniform(buffer_rsrc(base + int64_t(first) * ld, range32(bytes)));
    };
    auto load_tile = [&](const bf16_t* base, int64_t ld, const uint32_t* off, int j, uint32_t dst) {
      const u32x4 r = rows_of(base, ld, j);
#pragma unroll
      for (int i = 0; i < kL; ++i) lds_load16(dst, off[i], r, 0, 1024 * NW * i);
    };
    // Tiles' key blocks: those of the step and of the two after it.
    int j0 = walk.next(), j1 = n_tiles > 1 ? walk.next() : -1, j2 = -1;
    auto load_k = [&](int it, int j) {
      if (it < n_tiles) load_tile(K, a.k_ld, k_off, j, lds_w + (it & 1) * kTB);
    };
    auto load_v = [&](int it, int j) { load_tile(V, a.v_ld, v_off, j, lds_w + (2 + (it & 1)) * kTB); };

    const int sk = hi ^ swz_k(l32);
    // This lane's address for the transposed reads of V: row (l % 16) / 4 + 4 hi, column
    // 16 ((l / 16) % 2) + 4 (l % 4), less the tile and the 32-column group.
    const int vr = (lane % 16) / 4 + 4 * hi;
    const int va = vr * (DH * 2) + ((2 * ((lane / 16) % 2) + (lane % 4) / 2) ^ swz<DH>(vr)) * 16 + (lane % 2) * 8;
    typedef f32x16 STile[kKT / 32];
    typedef bf16x8 PTile[kKT / 16];
    constexpr int kQK = kC * (kKT / 32), kPV = kDT * (kKT / 16);
    constexpr int kRd = 4;  // fragments read ahead of their product
    auto fragment = [&](int i, int kbuf, int vbuf) {
      if (i >= kPV) {
        const int c = (i - kPV) / 2, t = (i - kPV) % 2;
        return as_bf16x8(*reinterpret_cast<const u32x4*>(smem + kbuf * kTB + (l32 + 32 * t) * (DH * 2) + ((2 * c) ^ sk) * 16));
      }
      const int c = i / kDT, dt = i % kDT;
      // Rows 16 c + 4 hi + .. and 8 more: the second's swizzle differs in bit 1 of the chunk.
      const int at = (va ^ (dt * 64)) + (2 + vbuf) * kTB + 16 * c * (DH * 2);
      const int at8 = (va ^ (dt * 64) ^ 32) + (2 + vbuf) * kTB + (16 * c + 8) * (DH * 2);
      const u32x2 lo = lds_read_tr(smem + at), up = lds_read_tr(smem + at8);
      return as_bf16x8(u32x4{lo[0], lo[1], up[0], up[1]});
    };
    auto product = [&](int i, const bf16x8& f, STile& sn, const PTile& pp) {
      if (i >= kPV) {
        const int c = (i - kPV) / 2, t = (i - kPV) % 2;
        sn[t] = mfma32(f, qf[c], c == 0 ? f32x16{} : sn[t]);
      } else {
        const int c = i / kDT, dt = i % kDT;
        oacc[dt] = mfma32(f, pp[c], oacc[dt]);
      }
    };
    // Keys past the sequence's last: logits to -inf.
    auto mask = [&](int j, STile& x) {
      const int up = s.k_hi - s.k_lo - j * kKB;
      if (up >= kKT) return;
      asm volatile("" ::: "memory");  // rare: a branch, not 32 selects on every tile
      const int u = up - 4 * hi;
#pragma unroll
      for (int t = 0; t < kKT / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * t + 8 * (r / 4) + r % 4 >= u) x[t][r] = -INFINITY;
    };
    // Logits of a tile to probabilities, without a branch, in slices: the row maximum over the first, then
    // the running maximum, then the exponentials and their sum.  corr is the
    // factor of the output so far (1 unless the maximum rose by more than 8).
    float corr = 1.f, ls = 0.f, mx = -INFINITY;
    auto softmax_slice = [&](int i, int n, STile& x, PTile& p) {
      const int n_max = n / 5, e0 = n_max + 1;
      if (i < n_max) {
        if (i == 0) mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (e >= 32 * i / n_max && e < 32 * (i + 1) / n_max) mx = fmaxf(mx, x[e / 16][e % 16]);
      } else if (i == n_max) {
        mx = max_xor32(mx) * scale2;
        const float m_new = mx > mrow + 8.f ? mx : mrow;
        corr = __builtin_amdgcn_exp2f(mrow - m_new);
        mrow = m_new;
        ls = 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          if (e < 32 * (i - e0) / (n - e0) || e >= 32 * (i + 1 - e0) / (n - e0)) continue;
          const float v = __builtin_amdgcn_exp2f(fmaf(x[e / 16][e % 16], scale2, -mrow));
          x[e / 16][e % 16] = v;
          ls += v;
          if (e % 2 == 1) {
            u32x4 w = __builtin_bit_cast(u32x4, p[e / 8]);
            w[(e % 8) / 2] = pack_bf2(x[e / 16][e % 16 - 1], v);
            p[e / 8] = as_bf16x8(w);
          }
        }
        if (i == n - 1) lrow = lrow * corr + ls;
      }
    };
    auto finish = [&]() {
      if (__any(corr != 1.f)) {
        asm volatile("" ::: "memory");  // rare: a branch, not a multiplication by 1 on every tile
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) oacc[dt] *= corr;
      }
    };
    // Slots [lo, up) of a step (the V fragments' products, then the K fragments') with the softmax of
    // (x, p) spread over them, in this order.
    // `loads(k)`, k < 2 kL, are spread over the first slots: issued together they hold up the wave, and the products
    // behind them, until the CU has taken them (1 KB in 16 cycles).
    auto run = [&](auto lo_tag, auto up_tag, auto soft_tag, int kbuf, int vbuf, STile& x, STile& sn, const PTile& pp, PTile& p,
                   auto loads) {
      constexpr int lo = decltype(lo_tag)::value, up = decltype(up_tag)::value;
      constexpr bool soft = decltype(soft_tag)::value;
      constexpr int n = up - lo > 10 ? up - lo : 10;  // slots
      bf16x8 f[kRd];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = lo; i < up && i < lo + kRd; ++i) f[(i - lo) % kRd] = fragment(i, kbuf, vbuf);
#pragma unroll
      for (int i = lo; i < lo + n; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if (i < up) {
          product(i, f[(i - lo) % kRd], sn, pp);
          if (i + kRd < up) f[(i - lo) % kRd] = fragment(i + kRd, kbuf, vbuf);
        }
        if ((i - lo) % 2 == 0 && (i - lo) / 2 < 2 * kL) loads((i - lo) / 2);
        if (soft) softmax_slice(i - lo, n, x, p);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    using Yes = std::integral_constant<bool, true>;
    using No = std::integral_constant<bool, false>;
    using Zero = std::integral_constant<int, 0>;
    using Pv = std::integral_constant<int, kPV>;
    using All = std::integral_constant<int, kQK + kPV>;
    auto step_barrier = [&]() {  // the loads issued one step ago have landed, for every wave
      vm_wait<0>();
      __builtin_amdgcn_sched_barrier(0);
      lds_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    auto none_on_its_way = [](int) {};
    STile sa, sb;
    PTile pa, pb;
    load_k(0, j0);
    load_k(1, j1);
    load_v(0, j0);
    if (n_tiles > 1) vm_wait<2 * kL>();
    else vm_wait<kL>();
    lds_barrier();
    run(Pv(), All(), No(), 0, 0, sb, sa, pa, pa, none_on_its_way);
    auto pin = [&](STile& sn, PTile& p) {  // the step's results are made in it, not sunk to where they are used
#pragma unroll
      for (int i = 0; i < kKT / 32; ++i) asm volatile("" : "+v"(sn[i]));
#pragma unroll
      for (int i = 0; i < kKT / 16; ++i) asm volatile("" : "+v"(p[i]));
#pragma unroll
      for (int i = 0; i < kDT; ++i) asm volatile("" : "+v"(oacc[i]));
      asm volatile("" : "+v"(lrow));
    };
    auto advance = [&](int t) {  // j0 = the key block of tile t
      j0 = j1;
      j1 = j2;
      j2 = t + 2 < n_tiles ? walk.next() : -1;
    };
    auto middle = [&](int t, int buf, STile& x, STile& sn, PTile& pp, PTile& p) {  // buf = (t - 1) & 1
      step_barrier();
      const bool more = t + 2 < n_tiles;
      u32x4 rk, rv;
      const uint32_t k_at = lds_w + (t & 1) * kTB, v_at = lds_w + (2 + (t & 1)) * kTB;
      mask(j1, x);
      run(Zero(), All(), Yes(), buf, buf, x, sn, pp, p, [&](int k) {
        if (k == 0) {
          advance(t);
          rv = rows_of(V, a.v_ld, j0);
          if (more) rk = rows_of(K, a.k_ld, j2);
        }
        if (k < kL) lds_load16(v_at, v_off[k], rv, 0, 1024 * NW * k);
        else if (more) lds_load16(k_at, k_off[k - kL], rk, 0, 1024 * NW * (k - kL));
      });
      pin(sn, p);
      finish();
    };
    step_barrier();
    j2 = n_tiles > 2 ? walk.next() : -1;
    load_k(2, j2);
    mask(j0, sa);
    if (n_tiles > 1) run(Pv(), All(), No(), 1, 0, sb, sb, pa, pa, none_on_its_way);
    run(Zero(), Zero(), Yes(), 0, 0, sa, sb, pa, pa, none_on_its_way);
    finish();
    if (n_tiles > 1) {
      int t = 1;
      for (; t + 2 < n_tiles; t += 2) {
        middle(t, 0, sb, sa, pa, pb);
        middle(t + 1, 1, sa, sb, pb, pa);
      }
      if (t + 1 < n_tiles) {
        middle(t, 0, sb, sa, pa, pb);
#pragma unroll
        for (int i = 0; i < kKT / 32; ++i) sb[i] = sa[i];
#pragma unroll
        for (int i = 0; i < kKT / 16; ++i) pa[i] = pb[i];
        ++t;
      }
      step_barrier();
      advance(t);
      load_v(t, j0);
      mask(j0, sb);
      run(Zero(), Pv(), Yes(), 0, (t - 1) & 1, sb, sa, pa, pb, none_on_its_way);
      finish();
#pragma unroll
      for (int i = 0; i < kKT / 16; ++i) pa[i] = pb[i];
    }
    step_barrier();
    run(Zero(), Pv(), No(), 0, (n_tiles - 1) & 1, sb, sa, pa, pb, none_on_its_way);
  }

  const float l = sum_xor32(lrow);
  if (row >= q_end) return;
  if (pieces > 1) {
    const int64_t at = sparse_slot(a, units, item.w, piece) * kQB + (row - q_first);
    float* po = a.part + at * DH + 4 * hi;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& o = oacc[dt];
        *reinterpret_cast<f32x4*>(po + 32 * dt + 8 * q) = f32x4{o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]};
      }
    if (hi == 0) reinterpret_cast<float2*>(a.part_ml)[at] = make_float2(mrow, l);
    return;
  }
  const bool none = walk.total == 0;
  if (a.lse && hi == 0) a.lse[int64_t(h) * a.M + row] = none ? -INFINITY : (mrow + log2f(l)) * kLn2;
  const float inv = none ? 0.f : 1.f / l;
  bf16_t* dst = static_cast<bf16_t*>(a.o) + int64_t(row) * a.o_ld + h * DH + 4 * hi;
#pragma unroll
  for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x16& o = oacc[dt];
      *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * q) =
          u32x2{pack_bf2(o[4 * q] * inv, o[4 * q + 1] * inv), pack_bf2(o[4 * q + 2] * inv, o[4 * q + 3] * inv)};
    }
}

// The pieces of each row joined in key order: with a piece's running maximum m_p, sum l_p and
// unnormalised output O_p, o = sum 2^(m_p - m) O_p / sum 2^(m_p - m) l_p, m the largest.  Eight pieces' loads
// are under way together.  Latency: 4 to 6.4 us (32 pieces).
template <int DH>
__global__ __launch_bounds__(256) void sparse_join_kernel(const SparseArgs a) {
  constexpr int kL = DH / 8, kR = 256 / kL, kPer = kQB / kR;  // lanes to a row, rows to a workgroup, workgroups to a unit
  const int units = a.seq.q_blk[kMaxSeqs] * a.H;
  const int4 cut = sparse_cut(a, blockIdx.x / kPer);
  if (cut.x < 0) return;
  const int blk = cut.x / a.H, h = cut.x % a.H, pieces = cut.y, r = blockIdx.x % kPer * kR + threadIdx.x / kL, c = threadIdx.x % kL * 8;
  const Seq s = seq_of<false>(a.seq, blk);
  const int row = s.q_lo + (blk - s.qb) * kQB + r;
  if (row >= s.q_hi) return;
  const int64_t step = sparse_slot(a, units, cut.z, 1) - cut.z, at = cut.z * int64_t(kQB) + r;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + at;
  const float* po = a.part + at * DH + c;
  float m = kNone, den = 0.f, acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int p0 = 0; p0 < pieces; p0 += 8) {
    float2 v[8];
    f32x4 x[8], y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t p = std::min(p0 + u, pieces - 1) * step * kQB;
      v[u] = ml[p];
      x[u] = *reinterpret_cast<const f32x4*>(po + p * DH);
      y[u] = *reinterpret_cast<const f32x4*>(po + p * DH + 4);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < 8; ++u) top = fmaxf(top, v[u].x);
    const float old = __builtin_amdgcn_exp2f(m - top);
    m = top;
    den *= old;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= old;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = p0 + u < pieces ? __builtin_amdgcn_exp2f(v[u].x - top) : 0.f;
      if (p0 + u >= pieces) continue;
      den = fmaf(w, v[u].y, den);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] = fmaf(w, x[u][e], acc[e]);
        acc[4 + e] = fmaf(w, y[u][e], acc[4 + e]);
      }
    }
  }
  const bool none = m == kNone && den == 0.f;  // no piece had a key
  if (a.lse && c == 0) a.lse[int64_t(h) * a.M + row] = none ? -INFINITY : (m + log2f(den)) * kLn2;
  const float inv = none ? 0.f : 1.f / den;
  *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(a.o) + int64_t(row) * a.o_ld + h * DH + c) =
      u32x4{pack_bf2(acc[0] * inv, acc[1] * inv), pack_bf2(acc[2] * inv, acc[3] * inv), pack_bf2(acc[4] * inv, acc[5] * inv),
            pack_bf2(acc[6] * inv, acc[7] * inv)};
}

// The plan of a forward pass alone.
__global__ __launch_bounds__(1024) void sparse_plan_kernel(const SparseArgs a, SparsePlan* plan) {
  __shared__ int counts[kMaxUnits];
  __shared__ uint64_t sums[1024];
  sparse_plan<false, 1024>(a, plan, counts, sums);
}

}  // namespace

template <int DH>
static void launch_forward(const SparseArgs& a, hipStream_t s) {
  const int64_t units = int64_t(a.seq.q_blk[kMaxSeqs]) * a.H;
  if (a.plan) hipLaunchKernelGGL(sparse_plan_kernel, dim3(1), dim3(1024), 0, s, a, const_cast<SparsePlan*>(a.plan));
  const int64_t n = a.plan ? units + a.slots : units * a.pieces, cuts = a.plan ? std::min<int64_t>(kShares, a.slots) : a.pieces > 1 ? units : 0;
  hipLaunchKernelGGL((sparse_bf16_kernel<DH>), dim3(unsigned(n)), dim3(256), 0, s, a);
  if (cuts > 0)
    hipLaunchKernelGGL((sparse_join_kernel<DH>), dim3(unsigned(cuts * (kQB * DH / 8 / 256))), dim3(256), 0, s, a);
}

void launch_sparse_bf16(const SparseArgs& a, hipStream_t s) {
  if (a.d == 128) launch_forward<128>(a, s);
  else launch_forward<64>(a, s);
}

}  // namespace avits
