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
#include "tiles.h"

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

// f(0) .. f(N - 1) with compile-time arguments.
template <typename F, int... I>
__device__ __forceinline__ void unrolled_over(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  unrolled_over(f, std::make_integer_sequence<int, N>());
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

// Few rows: a workgroup of NW waves owns 16 TM x 16 TN outputs, the waves take
// every NW-th step of the contraction straight from memory into registers (the next
// one while one is multiplied), and their sums meet in LDS.  Bound by the latency of a
// few loads in a row and the launch: 1 x 12288 x 2048 5.6 us in a graph for a weight of 13.4 MB.
template <int TM, int TN, int NW, typename T>
__global__ __launch_bounds__(64 * NW) void mx4_rows_kernel(const Mx4Args a) {
  __shared__ float red[NW][TM * TN * 4][kWave];
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
    struct Step {
      u32x4 x[TM][2], w[TN][2];
      Pairs<TM> sx;
      Pairs<TN> sw;
    };
    auto load = [&](int t, Step& v) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t c = uint32_t(t) * 128 + 32 * g + 16 * k;  // byte of the row; past its end nothing is read
#pragma unroll
        for (int j = 0; j < TN; ++j)
          v.w[j][k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                    rw, int(c < rowb ? (TN * l + j) * rowb + c : kNowhere), 0, 0));
#pragma unroll
        for (int i = 0; i < TM; ++i)
          v.x[i][k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                    rx, int(c < rowb ? (TM * l + i) * rowb + c : kNowhere), 0, 0));
      }
      const bool in = t < steps;
      v.sw = load_pairs<TN>(rws, in ? uint32_t(((4 * t + g) * Np + n0 + TN * l) * 2) : kNowhere);
      v.sx = load_pairs<TM>(rxs, in ? uint32_t(((4 * t + g) * Mp + m0 + TM * l) * 2) : kNowhere);
    };
    f32x4 acc[TM][TN] = {};
    Step cur, next;
    load(wave, cur);
    for (int t = wave; t < steps; t += NW) {
      load(t + NW, next);
      unrolled<2>([&](auto k) {
        unrolled<TM>([&](auto i) {
          unrolled<TN>([&](auto j) {
            acc[i][j] =
                mfma4<2 * (j % 2) + k, 2 * (i % 2) + k>(cur.w[j][k], cur.x[i][k], acc[i][j], cur.sw.v[j / 2], cur.sx.v[i / 2]);
          });
        });
      });
      cur = next;
    }
    // acc[i][j][r] = out[m0 + TM l + i][n0 + TN (4 g + r) + j].
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][(i * TN + j) * 4 + r][lane] = acc[i][j][r];
    __syncthreads();
    // The values of the tile, dealt over the waves.
    constexpr int kAll = TM * TN * 4;
    for (int v = wave; v < kAll; v += NW) {
      const int i = v / (TN * 4), j = v / 4 % TN, r = v % 4;
      float s = red[0][v][lane];
#pragma unroll
      for (int k = 1; k < NW; ++k) s += red[k][v][lane];
      const int64_t m = m0 + TM * l + i, n = n0 + TN * (4 * g + r) + j;
      if (m < a.M && n < a.N) finish<T>(a, m, n, s);
    }
    __syncthreads();  // before the next tile's sums
  }
}

// Sixteen consecutive elements, held as they lie in memory.
template <typename T>
struct Sixteen {
  static constexpr int V = int(sizeof(T));  // 16-byte words
  u32x4 w[V];
  __device__ __forceinline__ float at(int c) const {
    const uint32_t x = w[c * V / 16][c * V / 4 % 4];
    return V == 4 ? __uint_as_float(x) : __uint_as_float(c % 2 ? x & 0xffff0000u : x << 16);
  }
  // From element `first` of an array of `n` (zeros past its end), whatever its alignment.
  __device__ __forceinline__ void load(const void* base, int64_t n, int64_t first) {
    const __amdgpu_buffer_rsrc_t r = range_of(base, base ? n * int64_t(sizeof(T)) : 0);
#pragma unroll
    for (int c = 0; c < 4 * V; ++c) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t lo = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r, int((first + 2 * c) * 2), 0, 0));
        const uint32_t hi = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r, int((first + 2 * c + 1) * 2), 0, 0));
        w[c / 4][c % 4] = lo | hi << 16;
      } else {
        w[c / 4][c % 4] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(r, int((first + c) * 4), 0, 0));
      }
    }
  }
};

typedef const __attribute__((address_space(4))) Mx4Args* Mx4ArgsPtr;

// lds_load16 to LDS byte dst + OFF + 16 lane, the sum made in m0 itself.
template <int OFF>
__device__ __forceinline__ void lds_load16_at(uint32_t dst, uint32_t voff, const u32x4& rsrc, uint32_t soff) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               ::"s"(dst), "v"(voff), "s"(rsrc), "s"(soff), "n"(OFF) : "memory", "m0", "scc");
}
// Where 2 (bf16) or 4 (fp32) neighbouring lanes hold that many 16-byte chunks each
// of their own row, chunk q of lane p goes to lane q and comes back as its p:
// afterwards the lanes hold the chunks of one row side by side. (Its own inverse.)
template <int CTRL>
__device__ __forceinline__ void swap_chunks(u32x4& lower, u32x4& upper, bool is_upper) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t send = is_upper ? lower[e] : upper[e];
    const uint32_t got = uint32_t(__builtin_amdgcn_update_dpp(0, int(send), CTRL, 0xf, 0xf, false));
    lower[e] = is_upper ? got : lower[e];
    upper[e] = is_upper ? upper[e] : got;
  }
}
template <int V>
__device__ __forceinline__ void turn_chunks(u32x4 (&c)[V], int l) {
  if constexpr (V == 2) {
    swap_chunks<kDppXor1>(c[0], c[1], l & 1);
  } else {
    swap_chunks<kDppXor1>(c[0], c[1], l & 1);
    swap_chunks<kDppXor1>(c[2], c[3], l & 1);
    swap_chunks<kDppXor2>(c[0], c[2], l & 2);
    swap_chunks<kDppXor2>(c[1], c[3], l & 2);
  }
}

// The end of a 128 x 64 block that a wave holds as the tile kernel's sums: lane
// (l, g) has rows mb + 8 l + i and, of each, the columns nb + 16 g .. + 15.
// Whole 16-byte chunks of a row are turned over between neighbouring lanes, so
// that a store instruction covers whole rows of the block (16-byte pieces
// of 64 bytes each took four times as long): by buffer accesses that drop what lies
// outside, or (VEC false: rows or the bias do not start on 16 bytes) by plain ones,
// which may lie at any element, and a row's last, partial chunk one by one
// (4608 x 8195 x 2048 57.7 us, 8192 columns 55.4; column by column it took 164).
// A row's residual and gate are fetched before the row before it is stored: loads
// and stores complete in their order, so a wait for loads behind stores is one for the
// stores too (fp32 16896 x 2048 x 8192 504 us instead of 188, without a gate 150).
// BIAS_LDS: the block's biases lie in LDS.
template <typename T, bool GATED, bool VEC, bool BIAS_LDS>
struct BlockEnd {
  static constexpr int Z = sizeof(T), E = 16 / Z, V = 16 / E;   // elements of a chunk, chunks of a lane's columns
  Mx4ArgsPtr a;
  int64_t mb, nb, N;
  int l, g, rows, cols;
  bool one;
  const T* bias_lds;
  Sixteen<T> bias;
  __amdgpu_buffer_rsrc_t ro, rr;
  struct Fetched {
    Sixteen<T> resid, gate;
  };

  __device__ __forceinline__ BlockEnd(Mx4ArgsPtr args, int64_t mb_, int64_t nb_, int lane, const T* biases)
      : a(args), mb(mb_), nb(nb_), N(args->N), l(lane % 16), g(lane / 16),
        rows(int(std::min<int64_t>(128, args->M - mb_))), cols(int(std::min<int64_t>(64, args->N - nb_))),
        one(args->im.B == 1 || args->im.stride == 0), bias_lds(biases) {
    if (!BIAS_LDS) bias.load(a->bias, N, nb + 16 * g);
    else if (!GATED) bias_from_lds(bias);
    const int64_t span = ((rows - 1) * N + cols) * Z;
    ro = range_of(static_cast<T*>(a->out) + mb * N + nb, span);
    if (GATED) rr = range_of(static_cast<const T*>(a->resid) + mb * N + nb, span);
  }
  // Offset of chunk q after the turn: row 8 (l with its low bits q) + i, chunk V g + (l's low bits).
  __device__ __forceinline__ uint32_t at(int i, int q) const {
    const int chunk = V * g + (l & (V - 1)), row = 8 * ((l & ~(V - 1)) + q) + i;
    return E * chunk < cols ? uint32_t(row) * uint32_t(N * Z) + 16 * chunk : kNowhere;
  }
  // The same without alignment: where the chunk starts (elements of the output), and
  // how many of its elements there are (0: none).
  __device__ __forceinline__ int64_t loose_at(int i, int q, int& n) const {
    const int chunk = V * g + (l & (V - 1)), row = 8 * ((l & ~(V - 1)) + q) + i;
    n = row < rows ? std::max(0, std::min(E, cols - E * chunk)) : 0;
    return (mb + row) * N + nb + E * chunk;
  }
  __device__ __forceinline__ void bias_from_lds(Sixteen<T>& b) const {
#pragma unroll
    for (int q = 0; q < V; ++q)
      b.w[q] = a->bias ? *reinterpret_cast<const u32x4*>(bias_lds + 16 * g + E * q) : u32x4{0u, 0u, 0u, 0u};
  }
  // `n` elements of a chunk, zeros behind.
  static __device__ __forceinline__ u32x4 some(const T* p, int n) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (n >= E) {
      const loose4 c = *reinterpret_cast<const loose4*>(p);
      w = u32x4{c[0], c[1], c[2], c[3]};
    } else if (n > 0) {
#pragma unroll
      for (int e = 0; e < E - 1; ++e)
        if (e < n) w[e * Z / 4] |= element(p + e) << (Z == 2 && e % 2 ? 16 : 0);
    }
    return w;
  }
  __device__ __forceinline__ void fetch(int i, Fetched& f) const {
    if constexpr (GATED) {
      int64_t skip = 0;
      if (!one) {
        const int64_t stride = a->im.stride, at_row = mb + std::min(8 * l + i, rows - 1);
#pragma unroll 1
        for (int b = 0; b < a->im.B - 1; ++b) skip += at_row >= a->im.end[b] ? stride : 0;  // scalars are short: rolled
      }
      const T* gate = static_cast<const T*>(a->gate) + skip + nb + 16 * g;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        f.gate.w[q] = some(gate + E * q, cols - 16 * g - E * q);
        if constexpr (VEC) {
          f.resid.w[q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, int(at(i, q)), 0, 0));
        } else {
          int n;
          const T* p = static_cast<const T*>(a->resid) + loose_at(i, q, n);
          f.resid.w[q] = some(p, n);
        }
      }
    }
  }
  __device__ __forceinline__ void row(int i, float (&v)[16], Fetched& f) const {
    Sixteen<T> b = bias;
    if (BIAS_LDS && GATED) bias_from_lds(b);   // (registers are short)
#pragma unroll
    for (int c = 0; c < 16; ++c) v[c] += b.at(c);
    if constexpr (GATED) {
      turn_chunks<V>(f.resid.w, l);
#pragma unroll
      for (int c = 0; c < 16; ++c) v[c] = f.resid.at(c) + f.gate.at(c) * v[c];
    }
    u32x4 w[V];
#pragma unroll
    for (int q = 0; q < V; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[q][e] = Z == 4 ? __float_as_uint(v[4 * q % 16 + e]) : pack_bf2(v[(8 * q + 2 * e) % 16], v[(8 * q + 2 * e + 1) % 16]);
    turn_chunks<V>(w, l);
#pragma unroll
    for (int q = 0; q < V; ++q) {
      if constexpr (VEC) {
        __builtin_amdgcn_raw_buffer_store_b128(w[q], ro, int(at(i, q)), 0, 0);
      } else {
        int n;
        T* p = static_cast<T*>(a->out) + loose_at(i, q, n);
        if (n == E) {
          *reinterpret_cast<loose4*>(p) = loose4{w[q][0], w[q][1], w[q][2], w[q][3]};
        } else if (n > 0) {
#pragma unroll
          for (int e = 0; e < E - 1; ++e)
            if (e < n) {
              if constexpr (Z == 4) p[e] = __uint_as_float(w[q][e]);
              else p[e] = bf16_t(w[q][e / 2] >> (e % 2 ? 16 : 0));
            }
        }
      }
    }
  }
  static __device__ __forceinline__ uint32_t element(const T* p) {
    if constexpr (Z == 4) return __float_as_uint(*p);
    else return uint32_t(*p);
  }
};

// Many rows: 256 x 256 outputs to a workgroup of eight waves, a step of 256
// elements (128 bytes of every row) at a time.  In bytes and matrix cycles this
// is the bf16 product of a quarter of the contraction, and it runs in the same
// ping-pong form: two groups of four waves (one of each per SIMD), group g the
// output rows 128 g .. + 127, alternate a memory phase (read the fragments of a
// whole step from LDS, issue loads) with a compute phase (its 64 matrix
// instructions), one barrier per phase, the groups one phase apart:
//   phase 2t:     group 0 reads step t;        group 1 multiplies t - 1;
//   phase 2t + 1: group 0 multiplies step t;   group 1 reads t.
// Loads go to LDS directly.  Group 0 issues in phase 2t the first half of W and
// the second half of A (rows 128 .., which only group 1 reads) of step t + 1;
// group 1 in phase 2t + 1 the first half of A (read by group 0 only), the second
// half of W and the scales of step t + 2.  So two slots hold A, two the first half
// of W, three its second half and the scales, two the tile's
// biases: 158 KB.  LDS rows are 128 bytes;
// LDS row 16 i + l of a strip holds its row T l + i, block 2 g + k of a row lies
// in chunk (4 k + g) ^ (row / 2 mod 8): the 16 lanes that a read serves at once,
// of two lane groups, then meet every bank once (with the blocks in their own order
// half of them collided: 8192 x 8192 x 8192 took a twelfth longer).
// The contraction is short (8 steps for K = 2048), so a tile's head and tail
// are hidden too: a workgroup keeps taking tiles, the next tile's first loads go out before
// the stores of the last, and the waits for them leave those stores in flight.
// What bounds it: a phase takes about 1500 cycles instead of its 1024 of matrix
// instructions, since the fragments' reads and the loads' writes keep LDS busy for 1063
// of them, and a tile's end stores at HBM's rate.  8192 x 8192 x 8192 241 us (4.56
// PFLOP/s; matrix instructions alone reach 6.7), 16896 x 8192 x 2048 167 (3.39; its
// output alone 54 at a copy's rate), 4608 x 8192 x 2048 53, 1741 x 8192 x 2048 22.7.
// Four waves of 128 x 128 outputs, which read a third less from LDS, were slower (275 us
// and 208): with one wave per SIMD nothing runs beside its reads.
// PARTS: a tile is `splits` units, each a part of the contraction, and a unit's sums go
// to out as the registers lie: 16 bytes of every lane side by side, 256 KB a unit.
template <typename T, bool GATED, bool VEC, bool PARTS>
__global__ __launch_bounds__(512) void mx4_tile_kernel(const Mx4Args args, uint32_t units, uint32_t splits) {
  constexpr int TM = 8, TN = 4;
  // LDS in bytes: half a step of one operand is 16 KB.
  constexpr uint32_t kHalf = 0x4000, kA = 0, kWf = 4 * kHalf, kWs = 6 * kHalf, kS = 9 * kHalf, kSc = 0x1000, kB = kS + 3 * kSc;
  constexpr int kStores = PARTS ? 32 : TM * int(sizeof(T));   // store instructions of an epilogue of vectors
  __shared__ __attribute__((aligned(16))) char lds[kB + 2 * 1024];
  Mx4ArgsPtr a = (Mx4ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();  // scalar loads where needed
  const int tid = threadIdx.x;
  auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  auto uniform = [](u32x4 r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __builtin_amdgcn_readfirstlane(r[e]);
    return r;
  };
  auto bar = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  const int wave = scalar(tid / kWave);
  const int grp = wave / 4, sub = wave % 4;
  const uint32_t lds0 = uint32_t(scalar(int(uint32_t(reinterpret_cast<uintptr_t>(
      (__attribute__((address_space(3))) char*)(&lds[0]))))));
  const uint32_t rowb = uint32_t(a->K / 2), tn_all = uint32_t((a->N + 255) / 256), tm_all = uint32_t((a->M + 255) / 256);
  const int n_all = int((rowb + 127) / 128), n_whole = int(rowb / 128);

  // What a step needs per lane is made once: beside the matrix instructions of
  // the other group's wave every instruction of a memory phase costs its time.
  // One load instruction moves 8 LDS rows of 128 bytes; wave `sub` of a group
  // those from 8 sub + 32 j of a half (j = 0 .. 3).  LDS row r holds row T (r % 16)
  // + r / 16 of its strip; its chunk position p holds the block of slot p ^ (r / 2
  // mod 8), slot 4 k + g that of lane group g, k.
  uint32_t x_off[4], w_off[4];
  auto chunk_byte = [&](int lane) {   // byte of the row that the lane fetches
    const int slot = (lane % 8) ^ ((4 * sub + lane / 16) & 7);
    return uint32_t(16 * (2 * (slot & 3) + (slot >> 2)));
  };
  // LDS byte of a fragment within its strip's first tile, for k = 0 and 1, and
  // of the lane's scales.
  uint32_t f_at[2], s_at;
  {
    const int lane = tid % kWave, l = lane % 16, g = lane / 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = sub * 8 + lane / 8 + 32 * j;
      x_off[j] = uint32_t(128 * (1 - grp) + TM * (r % 16) + r / 16) * rowb + chunk_byte(lane);
      w_off[j] = uint32_t(128 * grp + 64 * (r / 64) + TN * (r % 16) + r / 16 % 4) * rowb + chunk_byte(lane);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) f_at[k] = 16 * (8 * l + ((4 * k + g) ^ ((l >> 1) & 7)));
    s_at = 512 * g + 16 * l;
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(x_off[j]), "+v"(w_off[j]));
    asm volatile("" : "+v"(f_at[0]), "+v"(f_at[1]), "+v"(s_at));
  }
  auto lane_id = []() { return int(__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u))); };
  // Scales: waves 0, 1 of group 1 load the rows' pairs (4 t + 2 sub, + 1), waves 2, 3 the columns'.
  const bool sc_w = sub >= 2;
  const uint32_t srow = uint32_t(scale_rows(sc_w ? a->N : a->M) * 2);

  // The tile in work: its place and where its loads start.
  int tm = 0, tn = 0, part = 0;
  int t0 = 0, n_t = 0;       // its first step, and how many it has
  u32x4 xr = {}, wr = {}, sr = {};
  uint32_t unit0 = 0;
  auto take = [&]() {   // the next tile of this workgroup; false: none
    while (unit0 < units) {
      const uint32_t here = unit0, n = std::min(units - here, uint32_t(gridDim.x));
      unit0 = here + n;
      if (blockIdx.x >= n) continue;
      int prob;
      const uint32_t unit = here + xcd_logical_id32(blockIdx.x, n);
      if (PARTS) part = scalar(int(unit));
      pp_place(unit / splits, tn_all, tm_all, 0, prob, tm, tn);
      tm = scalar(tm);
      tn = scalar(tn);
      t0 = scalar(int(uint32_t(n_all) * (unit % splits) / splits));
      n_t = scalar(int(uint32_t(n_all) * (unit % splits + 1) / splits)) - t0;
      const int64_t m0 = int64_t(tm) * 256, n0 = int64_t(tn) * 256;
      xr = uniform(buffer_rsrc(a->xq + m0 * rowb, uint32_t(std::min<int64_t>((a->M - m0) * rowb, kNowhere))));
      wr = uniform(buffer_rsrc(a->wq + n0 * rowb, uint32_t(std::min<int64_t>((a->N - n0) * rowb, kNowhere))));
      const int64_t skip = (sc_w ? n0 : m0) * 2;
      sr = uniform(buffer_rsrc((sc_w ? a->ws : a->xs) + skip, uint32_t(scale_groups(a->K) * srow - skip)));
      return true;
    }
    return false;
  };

  // The loads of step t (past the end: none of memory, but counted).
  auto load_half = [&](const u32x4& r, const uint32_t (&off)[4], uint32_t dst, int t) {
    const bool live = t < n_t;
    const u32x4 rr = {r[0], r[1], live ? r[2] : 0u, r[3]};
    const uint32_t k = live ? uint32_t(t0 + t) * 128 : 0u;
    if (t0 + t < n_whole) {
      lds_load16_at<0>(dst, off[0], rr, k);
      lds_load16_at<0x1000>(dst, off[1], rr, k);
      lds_load16_at<0x2000>(dst, off[2], rr, k);
      lds_load16_at<0x3000>(dst, off[3], rr, k);
    } else {   // the last step may end within a row's 128 bytes: what lies past them reads as 0
      const uint32_t far = k + chunk_byte(lane_id()) >= rowb ? kNowhere : 0u;
      lds_load16_at<0>(dst, off[0] | far, rr, k);
      lds_load16_at<0x1000>(dst, off[1] | far, rr, k);
      lds_load16_at<0x2000>(dst, off[2] | far, rr, k);
      lds_load16_at<0x3000>(dst, off[3] | far, rr, k);
    }
  };
  const uint32_t own = lds0 + sub * 1024;   // where this wave's rows of a half land
  auto load_a = [&](int t) { load_half(xr, x_off, own + kA + ((t & 1) * 2 + 1 - grp) * kHalf, t); };
  auto load_w = [&](int t, int slot3) {
    load_half(wr, w_off, own + (grp ? kWs + slot3 * kHalf : kWf + (t & 1) * kHalf), t);
  };
  auto load_s = [&](int t, int slot3) {
    const bool live = t < n_t;
    const u32x4 rr = {sr[0], sr[1], live ? sr[2] : 0u, sr[3]};
    const int lane = lane_id();
    const uint32_t off = (4 * uint32_t(t0 + t) + 2 * (sub & 1) + lane / 32) * srow + 16 * (lane % 32);
    lds_load16_at<0>(own + kS + slot3 * kSc, live ? off : kNowhere, rr, 0u);
  };

  f32x4 acc[TM][TN];
  u32x4 af[2][TM], wf[2][TN], as;
  u32x2 ws;
  const uint32_t w_first = (sub < 2 ? kWf : kWs) + (sub & 1) * 0x2000;
  auto read = [&](int t, int slot3) {
    const uint32_t A = kA + ((t & 1) * 2 + grp) * kHalf, W = w_first + (sub < 2 ? t & 1 : slot3) * kHalf, S = kS + slot3 * kSc;
    as = *reinterpret_cast<const u32x4*>(lds + S + grp * 256 + s_at);
    // (512 g + 8 l: four rows of a column pair array, s_at has eight.)
    ws = *reinterpret_cast<const u32x2*>(lds + S + 2048 + sub * 128 + (s_at & ~511u) + (s_at & 511u) / 2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int j = 0; j < TN; ++j) wf[k][j] = *reinterpret_cast<const u32x4*>(lds + W + f_at[k] + 2048 * j);
#pragma unroll
      for (int i = 0; i < TM; ++i) af[k][i] = *reinterpret_cast<const u32x4*>(lds + A + f_at[k] + 2048 * i);
    }
  };
  auto mul = [&]() {
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
    unrolled<2>([&](auto k) {
      unrolled<TM>([&](auto i) {
        unrolled<TN>([&](auto j) {
          acc[i][j] = mfma4<2 * (j % 2) + k, 2 * (i % 2) + k>(wf[k][j], af[k][i], acc[i][j], ws[j / 2], as[i / 2]);
        });
      });
    });
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  };

  int par = 0;               // which of two places the loads' tile has its biases in
  int64_t mb = -1, nb = 0;   // the finished tile's block of this wave
  int done = 0;              // and its unit
  for (;;) {
    // Every fragment of the finished tile has been read (group 0 is a barrier
    // past group 1's last read): the slots are free.  A wave's own late loads
    // past the end come before its next ones to the same place.
    asm volatile("" : "+s"(a));
    const bool more = take();
    if (more) {
      if (grp == 0) {
        // The tile's 256 biases (and what follows them), zeros past the end.
        if (VEC && a->bias)
          lds_load16_at<0>(lds0 + kB + 1024 * par, 16 * lane_id(),
                           uniform(buffer_rsrc(static_cast<const T*>(a->bias) + int64_t(tn) * 256,
                                               uint32_t((a->N - int64_t(tn) * 256) * int64_t(sizeof(T))))), 0u);
        load_w(0, 0);
        load_a(0);
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          load_a(t);
          load_w(t, t);
          load_s(t, t);
        }
      }
    }
    // acc[i][j][r] = out[mb + 8 l + i][nb + 16 g + 4 r + j].
    const bool out = mb >= 0 && mb < a->M && nb < a->N;
    if (out) {
      if constexpr (PARTS) {
        f32x4* p = static_cast<f32x4*>(a->out) + (int64_t(done) * 8 + wave) * (TM * TN * kWave) + lane_id();
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) p[(i * TN + j) * kWave] = acc[i][j];
      } else {
        using End = BlockEnd<T, GATED, VEC, VEC>;
        const End end(a, mb, nb, lane_id(), reinterpret_cast<const T*>(lds + kB + 1024 * (par ^ 1)) + 64 * sub);
        typename End::Fetched cur, nxt;
        end.fetch(0, cur);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if (i + 1 < TM) end.fetch(i + 1, nxt);
          float v[16];
#pragma unroll
          for (int c = 0; c < 16; ++c) v[c] = acc[i][c % 4][c / 4];
          end.row(i, v, cur);
          cur = nxt;
        }
      }
    }
    if (!more) break;
    par ^= 1;
    // Whether kStores stores at least are younger than the tile's first loads.
    int young = scalar(out && VEC ? 1 : 0);
    mb = int64_t(tm) * 256 + 128 * grp;
    nb = int64_t(tn) * 256 + 64 * sub;
    done = part;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (The step number and `young` are opaque: the loops would be peeled.)
    if (grp == 0) {
      if (young) vm_wait<4 + kStores>(); else vm_wait<4>();   // the first half of W(0)
      bar();
      int s3 = 0;
      for (int u = 0; u < n_t; ++u) {
        int t = u;
        asm volatile("" : "+s"(young), "+s"(t));
        read(t, s3);
        __builtin_amdgcn_sched_barrier(0);
        load_w(t + 1, 0);
        load_a(t + 1);
        // The second half of A(t), which phase 2t + 1 reads.
        if (young) vm_wait<8 + kStores>(); else vm_wait<8>();
        young >>= 1;
        bar();
        mul();
        vm_wait<4>();                 // the first half of W(t + 1), which phase 2t + 2 reads
        bar();
        s3 = s3 == 2 ? 0 : s3 + 1;
      }
    } else {
      if (young) vm_wait<9 + kStores>(); else vm_wait<9>();   // step 0
      bar();
      int s3 = 0;
      for (int u = 0; u < n_t; ++u) {
        int t = u;
        bar();
        asm volatile("" : "+s"(young), "+s"(t));
        const int s2 = s3 == 0 ? 2 : s3 - 1;   // the slot of t - 1 and t + 2
        read(t, s3);
        __builtin_amdgcn_sched_barrier(0);
        load_a(t + 2);
        load_w(t + 2, s2);
        load_s(t + 2, s2);
        // Step t + 1, which phase 2t + 2 reads.
        if (young) vm_wait<9 + kStores>(); else vm_wait<9>();
        young >>= 1;
        bar();
        mul();
        s3 = s3 == 2 ? 0 : s3 + 1;
      }
    }
  }
  vm_wait<0>();   // loads to LDS end before the workgroup does
}

// Joins the parts of a split product in their order: a workgroup a 128 x 64 block,
// a wave two of its eight row groups.
template <typename T, bool GATED, bool VEC>
__global__ __launch_bounds__(256) void mx4_join_kernel(const Mx4Args args, const float* __restrict__ parts, uint32_t splits) {
  const Mx4ArgsPtr a = (Mx4ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t tile = blockIdx.x / 8, block = blockIdx.x % 8;
  int prob, tm, tn;
  pp_place(tile, uint32_t((a->N + 255) / 256), uint32_t((a->M + 255) / 256), 0, prob, tm, tn);
  const int64_t mb = int64_t(tm) * 256 + 128 * (block / 4), nb = int64_t(tn) * 256 + 64 * (block % 4);
  if (mb >= a->M || nb >= a->N) return;
  using End = BlockEnd<T, GATED, VEC, false>;
  const End end(a, mb, nb, lane, nullptr);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = 2 * wave + h;
    typename End::Fetched f;
    end.fetch(i, f);
    f32x4 sum[4] = {};
    for (uint32_t k = 0; k < splits; ++k) {
      const f32x4* p = reinterpret_cast<const f32x4*>(parts) + ((int64_t(tile) * splits + k) * 8 + block) * (32 * kWave) +
                       i * 4 * kWave + lane;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += p[j * kWave];
    }
    float v[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) v[c] = sum[c % 4][c / 4];
    end.row(i, v, f);
  }
}

// The input gradient for few rows, straight from the held weight: a workgroup
// of NW waves owns 16 TM rows x 128 columns of dx, the waves take every NW-th 32
// rows n of W (the contraction) and their sums meet in LDS.  A lane loads 8 rows n =
// 8 g + e of W, 8 columns k = 8 l + t of each (one dword, one scale; the eight rows'
// scales lie side by side), turns them into bf16 (exact: e2m1 times a power of
// two) and has, for each t, the operand of one bf16 instruction: 8 n of column k.
// So the result's lane holds 8 consecutive columns of rows 4 g + r.
// Bound by the conversions (about 220 vector instructions for 8 TM matrix ones).
// ODD: N is no multiple of 8; dy's rows lie at any element, and of the last group of
// eight n what is not there counts as 0.
// An fp32 dy goes as three bf16 values whose sum it is exactly (8 bits of its 24 each), so
// their products with the weight's values are exact too and the sums are fp32's.  Only
// below 2^-110 can bits be left that lie under bf16's smallest, 2^-133: a wave that met
// some goes over its steps again and adds them as two more values, times 2^16, with the
// weight times 2^-16.  That is exact where it counts: a weight that 2^-16 takes below
// 2^-133 is at most 6 x 2^-117, and its product with such a rest is 0 in fp32.
// blockIdx.y: part of the contraction, summed into its own [M, K] where there are several.
struct Thirds {
  u32x4 v[3];
  uint32_t rest;   // its low half is not 0 where the three are less than the values
};
__device__ __forceinline__ Thirds thirds_of(const u32x4& lo, const u32x4& hi) {
  Thirds t;
  t.rest = 0;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t bits[3][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float x = __uint_as_float((e < 4 ? lo : hi)[e % 4 + h]);
      bits[0][h] = __float_as_uint(x) & 0xffff0000u;
      float r = x - __uint_as_float(bits[0][h]);
      r = __builtin_isinf(x) ? 0.f : r;   // (of NaN: NaN)
      bits[1][h] = __float_as_uint(r) & 0xffff0000u;
      bits[2][h] = __float_as_uint(r - __uint_as_float(bits[1][h]));
    }
    t.rest |= bits[2][0] | bits[2][1];
#pragma unroll
    for (int k = 0; k < 3; ++k) t.v[k][e / 2] = __builtin_amdgcn_perm(bits[k][1], bits[k][0], 0x07060302u);
  }
  return t;
}
// What the thirds leave, times 2^16: at most 16 bits from 2^-133 up, as two bf16 values.
__device__ __forceinline__ void rest_of(const u32x4& lo, const u32x4& hi, u32x4 (&v)[2]) {
  auto upper = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    uint32_t bits[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float r = __uint_as_float((e < 4 ? lo : hi)[e % 4 + h]);
      r = fabsf(r) < 0x1p-110f ? r : 0.f;
#pragma unroll
      for (int k = 0; k < 3; ++k) r -= upper(r);
      r *= 0x1p16f;
      bits[0][h] = __float_as_uint(upper(r));
      bits[1][h] = __float_as_uint(r - upper(r));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k][e / 2] = __builtin_amdgcn_perm(bits[k][1], bits[k][0], 0x07060302u);
  }
}

template <int TM, int NW, bool ODD, typename IN, typename OUT>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 4 : 1) void mx4_back_rows_kernel(
    const IN* __restrict__ dy, int64_t M, int64_t N, const uint8_t* __restrict__ wq, const uint8_t* __restrict__ ws, int64_t K,
    OUT* __restrict__ dx) {
  __shared__ float red[NW][TM * 32][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l = lane % 16, g = lane / 16;
  const int64_t tk = (K + 127) / 128;
  const int64_t k0 = int64_t(blockIdx.x) % tk * 128, m0 = int64_t(blockIdx.x) / tk * (16 * TM);
  const int64_t Np = scale_rows(N), rowb = K / 2, k = k0 + 8 * l;
  const __amdgpu_buffer_rsrc_t rs = range_of(ws, scale_groups(K) * Np * 2);
  constexpr int Z = sizeof(IN), V = Z / 2;   // 16-byte words of eight elements
  const __amdgpu_buffer_rsrc_t ry = range_of(dy + m0 * N, (M - m0) * N * Z);
  const int shift = 8 * int(k / 32 % 2);
  const int steps = int((N + 31) / 32);
  f32x4 acc[TM][8] = {};
  struct Step {
    uint32_t w[8];
    u32x4 sc, y[TM][V];
  };
  // (Past the last step everything is out of range: zeros, no memory.)
  // Byte offsets of the lane in the weight's 32 rows, its scales' and dy's rows (all below 2^31).
  struct At {
    uint32_t w, s, y;
  };
  const uint32_t row_bytes = uint32_t(rowb), n_all = uint32_t(N);
  auto place = [&](int l, int g) {
    const int64_t k = k0 + 8 * l;
    return At{k < K ? uint32_t(8 * g) * row_bytes + uint32_t(k / 2) : kNowhere, k < K ? uint32_t(k / 64 * Np * 2) : kNowhere,
              uint32_t(l) * n_all * Z};
  };
  auto load = [&](int t, Step& v, const At& p, int l, int g) {
    const uint32_t n = uint32_t(t) * 32 + 8 * g;
    const __amdgpu_buffer_rsrc_t rw = range_of(wq + int64_t(t) * 32 * rowb, (N - int64_t(t) * 32) * rowb);
    uint32_t at = p.w;
    asm volatile("" : "+v"(at));   // (eight offsets kept for the loop would spill)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v.w[e] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(rw, int(at + e * row_bytes), 0, 0));
    v.sc = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, int(n < n_all ? p.s + 2 * n : kNowhere), 0, 0));
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if constexpr (!ODD) {
#pragma unroll
        for (int q = 0; q < V; ++q)
          v.y[i][q] = __builtin_bit_cast(
              u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                         ry, int(n < n_all ? p.y + 16 * i * n_all * Z + n * Z + 16 * q : kNowhere), 0, 0));
      } else {   // (rows past M repeat the last one, unused)
        const IN* d = dy + std::min<int64_t>(m0 + 16 * i + l, M - 1) * N + n;
#pragma unroll
        for (int q = 0; q < V; ++q) {
          v.y[i][q] = u32x4{0u, 0u, 0u, 0u};
          if (n + 8 <= N) {
            const loose4 w = *reinterpret_cast<const loose4*>(d + 16 / Z * q);
            v.y[i][q] = u32x4{w[0], w[1], w[2], w[3]};
          }
        }
        if (n < N && n + 8 > N) {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (n + e < N) {
              if constexpr (Z == 4) v.y[i][e / 4][e % 4] = __float_as_uint(d[e]);
              else v.y[i][0][e / 2] |= uint32_t(d[e]) << (e % 2 ? 16 : 0);
            }
        }
      }
    }
    if (ODD && n < N && n + 8 > N) {   // (the codes past N read as 0; their scales may be anything)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e >= N) v.sc[e / 2] &= e % 2 ? 0xffffu : 0xffff0000u;
    }
  };
  const int stride = NW * int(gridDim.y);
  // The weight's columns of a step, times a power of two.
  auto decode = [&](const Step& v, float times, u32x4 (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      float a[8], b[8];
      const uint32_t pair = v.sc[e / 2] >> shift;
      decode4x8(v.w[e], scale_value(pair & 255u) * times, a);
      decode4x8(v.w[e + 1], scale_value(pair >> 16 & 255u) * times, b);
#pragma unroll
      for (int c = 0; c < 8; ++c) f[c][e / 2] = pack_bf2(a[c], b[c]);
    }
  };
  const int first = int(blockIdx.y) * NW + wave;
  uint64_t rest = 0;   // (of the wave: scalar)
  Step cur, next;
  const At here = place(l, g);
  load(first, cur, here, l, g);
  for (int t = first; t < steps; t += stride) {
    load(t + stride, next, here, l, g);
    u32x4 f[8];
    decode(cur, 1.f, f);
    if (Z == 4 && NW == 8) __builtin_amdgcn_sched_barrier(0);   // (128 registers hold no more at once)
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if constexpr (Z == 2) {
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[i][c] = mfma16x16x32(as_bf16x8(cur.y[i][0]), as_bf16x8(f[c]), acc[i][c]);
      } else {
        const Thirds y = thirds_of(cur.y[i][0], cur.y[i][1]);
        rest |= __ballot((y.rest & 0xffffu) != 0u);
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[i][c] = mfma16x16x32(as_bf16x8(y.v[k]), as_bf16x8(f[c]), acc[i][c]);
      }
    }
    cur = next;
  }
  auto put = [&](bool more) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float& at = red[wave][(i * 4 + r) * 8 + c][lane];
          at = more ? at + acc[i][c][r] : acc[i][c][r];
        }
  };
  put(false);
  if constexpr (Z == 4) {
    if (rest) {   // its steps again, for the rests
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      int l2 = l, g2 = g;
      asm volatile("" : "+v"(l2), "+v"(g2));   // (no registers for this loop's addresses in the one above)
      const At again = place(l2, g2);
#pragma unroll 1
      for (int t = first; t < steps; t += stride) {
        load(t, cur, again, l2, g2);
        u32x4 f[8];
        decode(cur, 0x1p-16f, f);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          u32x4 y[2];
          rest_of(cur.y[i][0], cur.y[i][1], y);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[i][c] = mfma16x16x32(as_bf16x8(y[k]), as_bf16x8(f[c]), acc[i][c]);
        }
      }
      put(true);
    }
  }
  __syncthreads();
  dx += int64_t(blockIdx.y) * M * K;
  // The 4 TM groups of eight columns of a lane, dealt over the waves.
  for (int v = wave; v < 4 * TM; v += NW) {
    float o[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      o[c] = red[0][v * 8 + c][lane];
#pragma unroll
      for (int u = 1; u < NW; ++u) o[c] += red[u][v * 8 + c][lane];
    }
    const int64_t m = m0 + 16 * (v / 4) + 4 * g + v % 4;
    if (m < M && k < K) store8(dx + m * K + k, o);
  }
}

// Sums of `parts` [n] arrays, in their order, in dx's type (n a multiple of 8).
template <typename T>
__global__ __launch_bounds__(256) void mx4_back_join_kernel(const float* __restrict__ part, int64_t n, int parts,
                                                            T* __restrict__ dx) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float v[8], t[8];
  load8(part + i, v);
  for (int k = 1; k < parts; ++k) {
    load8(part + k * n + i, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += t[e];
  }
  store8(dx + i, v);
}

// The weight as bf16 values, transposed: wt [K, ld] with zeros in columns N .. ld.
// A lane takes 8 rows n x 8 columns k (a dword each, as in the kernel above) and has,
// for each k, 16 bytes of a row of wt; a wave covers 64 n x 64 k, a workgroup 64 x
// 256, so that both sides move 128 bytes of a row.  8192 x 2048: 10.1 us for 42
// MB (through LDS 14.1), beside 138 of the product of 4608 rows.
__global__ __launch_bounds__(256) void transpose4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                         int64_t N, int64_t K, bf16_t* __restrict__ wt, int64_t ld) {
  const int lane = threadIdx.x % kWave;
  const int64_t n = int64_t(blockIdx.x) * 64 + 8 * (lane % 8);
  const int64_t k = int64_t(blockIdx.y) * 256 + 64 * (threadIdx.x / kWave) + 8 * (lane / 8);
  if (k >= K) return;
  uint32_t w[8] = {};
  u32x4 sc = {0u, 0u, 0u, 0u};
  if (n < N) {
    sc = *reinterpret_cast<const u32x4*>(s + (k / 64 * scale_rows(N) + n) * 2);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < N) w[e] = *reinterpret_cast<const uint32_t*>(q + ((n + e) * K + k) / 2);
  }
  const int shift = 8 * int(k / 32 % 2);
  u32x4 f[8];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float a[8], b[8];
    const uint32_t pair = sc[e / 2] >> shift;   // (rows past N may have any scale)
    decode4x8(w[e], n + e < N ? scale_value(pair & 255u) : 0.f, a);
    decode4x8(w[e + 1], n + e + 1 < N ? scale_value(pair >> 16 & 255u) : 0.f, b);
#pragma unroll
    for (int c = 0; c < 8; ++c) f[c][e / 2] = pack_bf2(a[c], b[c]);
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) *reinterpret_cast<u32x4*>(wt + (k + c) * ld + n) = f[c];
}

// Rows of N elements to rows of ld (a multiple of 64), zeros behind: 16 bytes a lane,
// read at any element.
__global__ __launch_bounds__(256) void widen_kernel(const bf16_t* __restrict__ x, int64_t M, int64_t N,
                                                    bf16_t* __restrict__ y, int64_t ld) {
  constexpr int E = 8;
  const int64_t n = (int64_t(blockIdx.y) * 64 + threadIdx.x % 64) * E;
  if (n >= ld) return;
  for (int64_t m = int64_t(blockIdx.x) * 4 + threadIdx.x / 64; m < M; m += int64_t(gridDim.x) * 4) {
    const bf16_t* p = x + m * N + n;
    u32x4 w = {0u, 0u, 0u, 0u};
    if (n + E <= N) {
      const loose4 v = *reinterpret_cast<const loose4*>(p);
      w = u32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < E - 1; ++e)
        if (n + e < N) w[e / 2] |= uint32_t(p[e]) << (e % 2 ? 16 : 0);
    }
    *reinterpret_cast<u32x4*>(y + m * ld + n) = w;
  }
}

int check_product(const char* who, int64_t M, int64_t N, int64_t K, int dtype) {
  AVITS_REQUIRE(M >= 0 && M < (int64_t(1) << 27), "%s: M=%lld outside [0, 2^27)", who, (long long)M);
  AVITS_REQUIRE(N >= 1 && N < (int64_t(1) << 21), "%s: N=%lld outside [1, 2^21)", who, (long long)N);
  AVITS_REQUIRE(K >= kBlk && K < (int64_t(1) << 21) && K % kBlk == 0, "%s: K=%lld must be a multiple of 32 in [32, 2^21)", who,
                (long long)K);
  AVITS_REQUIRE(scale_groups(K) * scale_rows(std::max(M, N)) * 2 < (int64_t(1) << 31),
                "%s: %lld x %lld has 2^31 scales or more", who, (long long)std::max(M, N), (long long)K);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  return AVITS_OK;
}

// How a product runs: 256 x 256 tiles, each in `splits` parts of the contraction,
// or (splits == 0) form `rows` of the kernel for few rows.  The least predicted
// time (us), from what was measured:
//  - few rows: the largest of the operands' bytes, which each workgroup reads for
//    itself, at the rate its form reaches, its chain of steps over its waves, and the
//    outputs, stored one by one (16000 x 8192 x 96: 539 us; by tiles 60);
//  - tiles, in equal rounds of at most one unit per CU: 1.2 (few CUs busy) to 1.5 a
//    step and 6.5 a unit; parts are written and read at 7 TB/s by a second launch.
// Measured (bf16 out; forms 1 x 1, 2 x 2, 4 x 2, 4 x 4 strips of 16, tiles whole, in 4 parts):
//   16 x 8192 x 2048    5.5   5.0   6.2  10.3  15.6  21.5     32 x 2048 x 8192     7.0  11.8  13.7  21.1  45.5  23.1
//   64 x 8192 x 2048   14.6   8.7   8.2  12.5  15.7  21.6     300 x 4096 x 4096   42.5  25.8  28.5  24.6  26.7  26.9
//   512 x 8192 x 2048  93.1  49.4  51.5  35.1  17.9  32.1     1741 x 2048 x 8192   214   112   103  75.5  47.5  36.9
constexpr struct {
  int tm, tn, waves;
  double fixed, rate, step;   // us beside, TB/s from the caches, us a step of the chain
} kForms[4] = {{1, 1, 8, 2.5, 7.0, 1.1}, {2, 2, 8, 2.5, 7.0, 2.3}, {4, 2, 8, 3.5, 6.0, 2.6}, {4, 4, 4, 6.0, 4.8, 2.0}};
struct ProductPlan {
  int splits = 0, form = 0;
};
constexpr size_t kMaxPartBytes = size_t(64) << 20;
constexpr int kCUs = 256, kMaxSplits = 4;
size_t part_bytes(int splits, int64_t M, int64_t N) {
  return size_t(splits) * size_t(ceil_div64(M, 256)) * size_t(ceil_div64(N, 256)) * (256 * 256 * sizeof(float));
}
ProductPlan plan_product(int64_t M, int64_t N, int64_t K) {
  ProductPlan p;
  const double steps = double(ceil_div64(K, kStepK));
  double best = 1e30;
  for (int f = 0; f < 4; ++f) {
    const auto& form = kForms[f];
    const double wgs = double(ceil_div64(M, 16 * form.tm)) * double(ceil_div64(N, 16 * form.tn));
    const double bytes = wgs * 16.0 * (form.tm + form.tn) * double(K) * 0.53e-6;
    const double us = form.fixed + std::max({bytes / form.rate, std::ceil(steps / form.waves) * form.step,
                                             double(M) * double(N) * 3.8e-6});
    if (us >= best) continue;
    best = us;
    p.form = f;
  }
  const double tiles = double(ceil_div64(M, 256)) * double(ceil_div64(N, 256));
  for (int sp = 1; sp <= kMaxSplits && sp <= int(steps); ++sp) {
    if (sp > 1 && part_bytes(sp, M, N) > kMaxPartBytes) break;
    const double units = tiles * sp, rounds = std::ceil(units / kCUs), per = std::ceil(units / rounds);
    const double us = rounds * (std::ceil(steps / sp) * (1.2 + 0.3 * per / kCUs) + 6.5) +
                      (sp > 1 ? 3.0 + 2e-6 * double(part_bytes(sp, M, N)) / 7.0 : 0.0);
    if (us >= best) continue;
    best = us;
    p.splits = sp;
  }
  return p;
}

template <typename T>
void run_product(const Mx4Args& a, const ProductPlan& p, float* part, hipStream_t s) {
  TimedLaunch timed("mxfp4_linear", s);
  auto rows = [&](auto tm, auto tn, auto nw) {
    constexpr int kTM = decltype(tm)::value, kTN = decltype(tn)::value, kNW = decltype(nw)::value;
    const int64_t tiles = ceil_div64(a.M, 16 * kTM) * ceil_div64(a.N, 16 * kTN);
    hipLaunchKernelGGL((mx4_rows_kernel<kTM, kTN, kNW, T>), dim3(unsigned(std::min<int64_t>(tiles, 1 << 22))), dim3(64 * kNW), 0,
                       s, a);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  const integral_constant<int, 4> four;
  const integral_constant<int, 8> eight;
  if (p.splits == 0) {
    if (p.form == 0) rows(one, one, eight);
    else if (p.form == 1) rows(two, two, eight);
    else if (p.form == 2) rows(four, two, eight);
    else rows(four, four, four);
    return;
  }
  const int64_t units = ceil_div64(a.M, 256) * ceil_div64(a.N, 256) * p.splits;
  const dim3 grid(unsigned(ceil_div64(units, ceil_div64(units, kCUs)))), wg(512);
  const bool vec = a.N % (16 / int64_t(sizeof(T))) == 0 && aligned_to({a.bias}, 16);
  auto by_form = [&](auto go) {
    const std::true_type yes;
    const std::false_type no;
    if (a.gate && vec) go(yes, yes);
    else if (a.gate) go(yes, no);
    else if (vec) go(no, yes);
    else go(no, no);
  };
  if (p.splits == 1) {
    by_form([&](auto gated, auto vectors) {
      hipLaunchKernelGGL((mx4_tile_kernel<T, decltype(gated)::value, decltype(vectors)::value, false>), grid, wg, 0, s, a,
                         uint32_t(units), 1u);
    });
    return;
  }
  Mx4Args g = a;
  g.bias = nullptr;
  g.out = part;
  hipLaunchKernelGGL((mx4_tile_kernel<float, false, true, true>), grid, wg, 0, s, g, uint32_t(units), uint32_t(p.splits));
  by_form([&](auto gated, auto vectors) {
    hipLaunchKernelGGL((mx4_join_kernel<T, decltype(gated)::value, decltype(vectors)::value>),
                       dim3(unsigned(units / p.splits * 8)), dim3(256), 0, s, a, (const float*)part, uint32_t(p.splits));
  });
}

// Scratch of the input gradient (bf16): the weight transposed, dy widened where its
// rows are not whole contraction tiles, and split sums of the product; or parts.
struct BackPlan {
  int64_t ld;
  size_t wt = 0, dy = 0, part = 0;
  int rows = 0, parts = 1;   // rows > 0: the kernel for few rows with 16 `rows` rows to a workgroup
};
// Few rows (bf16) go straight from the held weight, 16 of them to a workgroup of eight
// waves (two of which fit a CU) or 64 to one of four, the contraction whole or in
// parts; the other way is to turn the weight round and run the bf16 product.  The
// least predicted time (us).  A chain step takes 1.0 us (1.7 with two workgroups on a
// CU; 1.2 with 64 rows), parts their bytes and a launch, which the host pays too; the
// other way its launches, the weight's bytes and the product at 1.1 PFLOP/s.  fp32
// always goes from the held weight, by the same figures (within 8 % of its best form from
// 300 x 2051 x 2048, 24.9 us in a graph, to 1741 x 6400 x 2048, 176-182; 1 x 1024 x 1024 8.2 and in 4
// parts 6.8, whose second launch the host would pay; the fp32 product with the
// weight turned round took 13.1 and 723).  Measured (16 rows whole, in 4; 64 rows in 4; turned round):
//   16 x 8192 x 2048   30.3  12.7  21.6  44.8     512 x 8192 x 2048  58.6  60.0  53.6  44.0
//   128 x 8192 x 2048  31.4  21.2  28.5  41.5     67 x 1024 x 256     6.7   6.8   9.7  14.2
//   256 x 8192 x 2048  33.8  34.7  30.4  41.2     64 x 2048 x 8192   11.2  18.0  15.9  31.0
//   300 x 2051 x 2048  19.3  22.2  26.2  32.7     1741 x 1024 x 512  10.3  19.9  21.0  24.2
BackPlan plan_back(int64_t M, int64_t N, int64_t K, int dtype) {
  const bool half = dtype == AVITS_BF16;
  BackPlan p;
  p.ld = ceil_div64(N, 64) * 64;
  if (half) {
    p.wt = align_up(size_t(K) * size_t(p.ld) * 2, 256);
    p.dy = p.ld != N ? align_up(size_t(M) * size_t(p.ld) * 2, 256) : 0;
    p.part = std::min<size_t>(gemm_partial_reserve(M, K), size_t(64) << 20);
  }
  const double weights = double(N) * double(K) * 1e-6;
  double best = half ? (p.dy ? 22.0 : 16.0) + weights * 4.5 / 5.0 + 2.0 * double(M) * weights / 1.1e3 : 1e30;
  for (int rows : {1, 4})
    for (int parts = 1; parts <= 8; parts *= 2) {
      const int waves = rows == 1 ? 8 : 4;
      const int64_t steps = ceil_div64(N, 32), wgs = ceil_div64(M, 16 * rows) * ceil_div64(K, 128) * parts;
      if (parts > 1 && (steps < parts * waves || size_t(parts) * size_t(M) * size_t(K) * sizeof(float) > kMaxPartBytes)) break;
      const double step = rows == 4 ? 1.2 : wgs <= kCUs ? 1.0 : 1.7;
      const double us = 2.5 + double(ceil_div64(steps, waves * parts)) * step * double(ceil_div64(wgs, rows == 4 ? kCUs : 2 * kCUs)) +
                        (parts > 1 ? 3.5 + double(parts) * double(M) * double(K) * 8e-6 / 4.0 : 0.0);
      if (us >= best) continue;
      best = us;
      p.rows = rows;
      p.parts = parts;
    }
  return p;
}

// dx by mx4_back_rows_kernel, as the plan says.
template <typename T>
int run_back_rows(const BackPlan& p, const T* dy, int64_t M, int64_t N, const uint8_t* wq, const uint8_t* ws, int64_t K, T* dx,
                  float* part, hipStream_t s) {
  TimedLaunch timed("mxfp4_backward", s);
  auto go = [&](auto tm, auto nw, auto* out) {
    constexpr int kTM = decltype(tm)::value, kNW = decltype(nw)::value;
    using Out = std::remove_pointer_t<decltype(out)>;
    const dim3 grid(unsigned(ceil_div64(M, 16 * kTM) * ceil_div64(K, 128)), unsigned(p.parts));
    if (N % 8 == 0)
      hipLaunchKernelGGL((mx4_back_rows_kernel<kTM, kNW, false, T, Out>), grid, dim3(64 * kNW), 0, s, dy, M, N, wq, ws, K, out);
    else
      hipLaunchKernelGGL((mx4_back_rows_kernel<kTM, kNW, true, T, Out>), grid, dim3(64 * kNW), 0, s, dy, M, N, wq, ws, K, out);
  };
  using std::integral_constant;
  auto by_rows = [&](auto* out) {
    if (p.rows == 1) go(integral_constant<int, 1>(), integral_constant<int, 8>(), out);
    else go(integral_constant<int, 4>(), integral_constant<int, 4>(), out);
  };
  if (p.parts == 1) {
    by_rows(dx);
  } else {
    by_rows(part);
    hipLaunchKernelGGL(mx4_back_join_kernel<T>, dim3(unsigned(ceil_div64(M * K / 8, 256))), dim3(256), 0, s, (const float*)part,
                       M * K, p.parts, dx);
  }
  return launch_status("mxfp4_linear_backward");
}

// dx by the bf16 product with the weight turned round.
int run_back_tiles(const BackPlan& p, const bf16_t* dy, int64_t M, int64_t N, const uint8_t* wq, const uint8_t* ws, int64_t K,
                   bf16_t* dx, char* scratch, hipStream_t s) {
  bf16_t* wt = reinterpret_cast<bf16_t*>(scratch);
  {
    TimedLaunch timed("mxfp4_transpose", s);
    hipLaunchKernelGGL(transpose4_kernel, dim3(unsigned(p.ld / 64), unsigned(ceil_div64(K, 256))), dim3(256), 0, s, wq, ws, N, K,
                       wt, p.ld);
    if (p.dy) {
      bf16_t* wide = reinterpret_cast<bf16_t*>(scratch + p.wt);
      hipLaunchKernelGGL(widen_kernel, dim3(unsigned(std::min<int64_t>(ceil_div64(M, 4), 4096)), unsigned(ceil_div64(p.ld, 512))),
                         dim3(256), 0, s, dy, M, N, wide, p.ld);
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
  return launch_gemm(g, AVITS_BF16, s, "mxfp4_backward", p.part ? reinterpret_cast<float*>(scratch + p.wt + p.dy) : nullptr,
                     p.part);
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" size_t avits_mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (check_product("mxfp4_linear_workspace_bytes", M, N, K, AVITS_BF16) != AVITS_OK || M == 0) return 0;
  const int64_t steps = ceil_div64(K, kStepK);
  return steps < 2 ? 0 : std::min(kMaxPartBytes, part_bytes(int(std::min<int64_t>(steps, kMaxSplits)), M, N));
}

extern "C" int avits_mxfp4_linear(const uint8_t* xq, const uint8_t* xs, int64_t M, int64_t K, const uint8_t* wq,
                                  const uint8_t* ws, const void* b, int64_t N, int32_t B, const int64_t* off,
                                  const void* gate, int64_t mod_stride, const void* resid, int dtype, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_product("mxfp4_linear", M, N, K, dtype);
  Mx4Args a = {xq, xs, wq, ws, b, gate, resid, out, M, N, K, {}};
  if (rc == AVITS_OK) rc = fill_images("mxfp4_linear", M, B, off, mod_stride, a.im);
  if (rc != AVITS_OK) return rc;
  if (M == 0) return AVITS_OK;
  AVITS_REQUIRE((gate != nullptr) == (resid != nullptr), "mxfp4_linear: gate and resid go together");
  AVITS_REQUIRE(xq && xs && wq && ws && out, "mxfp4_linear: null xq/xs/wq/ws/out");
  AVITS_REQUIRE(aligned_to({xq, xs, wq, ws, out, resid}, 16),
                "mxfp4_linear: xq, xs, wq, ws, resid and out must be 16-byte aligned");
  AVITS_REQUIRE(aligned_to({b, gate}, dtype == AVITS_BF16 ? 2 : 4), "mxfp4_linear: b or gate is not aligned to its element");
  const ProductPlan p = plan_product(M, N, K);
  const size_t need = p.splits > 1 ? part_bytes(p.splits, M, N) : 0;
  if (need && (!workspace || workspace_bytes < need))
    return set_error(AVITS_ERR_WORKSPACE, "mxfp4_linear: workspace of %zu bytes, need %zu", workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  AVITS_REQUIRE(!need || aligned_to({workspace}, 16), "mxfp4_linear: workspace must be 16-byte aligned");
  if (dtype == AVITS_BF16) run_product<bf16_t>(a, p, static_cast<float*>(workspace), s);
  else run_product<float>(a, p, static_cast<float*>(workspace), s);
  return launch_status("mxfp4_linear");
}

extern "C" size_t avits_mxfp4_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int dtype) {
  if (check_product("mxfp4_linear_backward_workspace_bytes", M, N, K, dtype) != AVITS_OK) return 0;
  const BackPlan p = plan_back(M, N, K, dtype);
  // Any smaller M too, which may run as parts of [M, K] (at most 64 MiB of them).
  const size_t few = std::min<size_t>(kMaxPartBytes, size_t(8) * size_t(M) * size_t(K) * sizeof(float));
  return std::max(p.wt + p.dy + p.part, few);
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
  const BackPlan p = plan_back(M, N, K, dtype);
  float* part = static_cast<float*>(workspace);
  if (dtype == AVITS_F32)
    return run_back_rows(p, static_cast<const float*>(dy), M, N, wq, ws, K, static_cast<float*>(dx), part, s);
  const bf16_t* y = static_cast<const bf16_t*>(dy);
  bf16_t* x = static_cast<bf16_t*>(dx);
  rc = p.rows ? run_back_rows(p, y, M, N, wq, ws, K, x, part, s) : run_back_tiles(p, y, M, N, wq, ws, K, x, scratch, s);
  return rc != AVITS_OK ? rc : launch_status("mxfp4_linear_backward");
}
