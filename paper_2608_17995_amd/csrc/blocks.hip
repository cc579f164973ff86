// Which key blocks each query block attends to: the mean of every block of
// queries and of keys, the products of the means, and of each query block's scores
// the best.
//
// Means, scores and comparisons are in 64 bits: the choice is then that of the
// formula, whatever the order of the sums, except among scores that agree to some
// fifteen digits.
#include "sparse.h"

namespace avits {

int seq_rows(const char* what, int32_t B, const int64_t* off, int64_t rows, int block, int32_t* row, int32_t* blk) {
  AVITS_REQUIRE(B >= 1 && B <= kMaxSeqs, "%s: B=%d outside [1, %d]", what, B, kMaxSeqs);
  AVITS_REQUIRE(rows >= 0 && rows < (int64_t(1) << 31) - 4096, "%s: %lld rows outside [0, 2^31 - 4096)", what, (long long)rows);
  AVITS_REQUIRE(off || B == 1, "%s: no offsets for %d sequences", what, B);
  row[0] = 0;
  blk[0] = 0;
  for (int b = 0; b < B; ++b) {
    const int64_t lo = off ? off[b] : 0, hi = off ? off[b + 1] : rows;
    AVITS_REQUIRE((b > 0 || lo == 0) && hi >= lo && hi <= rows, "%s: offsets must rise from 0 to at most %lld", what, (long long)rows);
    row[b + 1] = int32_t(hi);
    blk[b + 1] = blk[b] + int32_t((hi - lo + block - 1) / block);
  }
  return AVITS_OK;
}

int seq_blocks(SeqBlocks& s, const char* what, int32_t B, const int64_t* q_off, int64_t M, const int64_t* k_off, int64_t N) {
  s = SeqBlocks{};
  s.B = B;
  int rc = seq_rows(what, B, q_off, M, kQB, s.q_row, s.q_blk);
  if (rc == AVITS_OK) rc = seq_rows(what, B, k_off, N, kKB, s.k_row, s.k_blk);
  return rc;
}

namespace {

// ---------------------------------------------------------------------------
// Means.  A workgroup takes one block and 32 vectors of 16 bytes of its columns;
// eight strands of rows meet in LDS.  Bound by reading x once: 16896 rows of 16 heads of 128 in bf16, 69 MB, 10.8 to
// 13.4 us, 5.1 TB/s and more with what the caches still hold.
struct MeanArgs {
  const void* x;
  int64_t ld;
  double* out;
  int32_t B, block, blocks, cols;
  int32_t row[kMaxSeqs + 1], blk[kMaxSeqs + 1];
};

template <typename T>
__global__ __launch_bounds__(256) void block_means_kernel(const MeanArgs a) {
  constexpr int kV = 16 / sizeof(T);  // columns to a thread
  __shared__ double red[8][kV][33];
  const int vec = threadIdx.x % 32, strand = threadIdx.x / 32, blk = int(wide_block());
  const int col = (blockIdx.z * 32 + vec) * kV;
  if (blk >= a.blocks) return;
  int lo = a.row[0], hi = a.row[1], b0 = 0;
#pragma unroll
  for (int b = 1; b < kMaxSeqs; ++b)
    if (b < a.B && blk >= a.blk[b]) lo = a.row[b], hi = a.row[b + 1], b0 = a.blk[b];
  lo += (blk - b0) * a.block;
  const int n = std::min(a.block, hi - lo);
  double acc[kV];
#pragma unroll
  for (int e = 0; e < kV; ++e) acc[e] = 0.0;
  if (col < a.cols) {
    const T* src = static_cast<const T*>(a.x) + int64_t(lo) * a.ld + col;
#pragma unroll 8
    for (int r = strand; r < n; r += 8) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(src + r * a.ld);
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        if constexpr (sizeof(T) == 4) acc[e] += double(__uint_as_float(w[e]));
        else acc[e] += double(__uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16));
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kV; ++e) red[strand][e][vec] = acc[e];
  __syncthreads();
  // 32 kV columns by 256 threads: one (fp32: half the threads) column each.
  const int e = threadIdx.x % kV, v = threadIdx.x / kV;
  if (v >= 32) return;
  double sum = 0.0;
#pragma unroll
  for (int s = 0; s < 8; ++s) sum += red[s][e][v];
  const int c = (blockIdx.z * 32 + v) * kV + e;
  if (c < a.cols) a.out[int64_t(blk) * a.cols + c] = sum / n;
}

// ---------------------------------------------------------------------------
// Scores and choice.  A workgroup takes up to 16 query blocks of a head of one
// sequence: their scores against all key blocks by 16x16x4 products in 64 bits into
// LDS, then a wave for each row finds the n-th largest by its bits, from the highest, with the keys in registers
// where there are at most 512.
// Times at 264 key blocks, 132 query blocks and 16 heads of 128: keys read from LDS for each bit 42 us, from registers 30;
// the products' operands fetched as a lane needs them, 64 bytes of each of 16 rows to an instruction, kept the L1
// cache busy for 20 us of these: a row's bytes are now fetched together and change lanes in LDS (20 us).  Of these the
// counting takes 6 (up to 64 rounds, each of which needs the last), the products 4, the fetch of the keys' means 2; the other 8 are
// the start, the queries' means and the mask's words.
constexpr int kSelWaves = 8;
constexpr int kMaxKeyBlocks = 16384;  // 128 KiB of scores for one row

struct SelectArgs {
  const double *qm, *km;
  uint64_t* mask;
  SeqBlocks seq;
  int64_t words;
  int H, Hk, d, rows;   // rows: query blocks to a workgroup
  int q_lead, k_lead, keep;
  int groups[kMaxSeqs + 1];  // workgroups (of a head) before each sequence; all of them in the last entry
};

typedef double f64x2 __attribute__((ext_vector_type(2)));
typedef double f64x4 __attribute__((ext_vector_type(4)));

// Order-preserving: NaN below every number, -0 as +0.
__device__ __forceinline__ uint64_t order_key(double v) {
  if (v != v) return 0;
  const uint64_t u = uint64_t(__double_as_longlong(v + 0.0));
  return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}

// The choice of one row by a wave: key(t) is the ordered score of key block 64 t + lane, 0 for those that do not
// compete (the leading ones, and past the last).  HELD: the number of tiles, from registers (0: any).
template <int HELD, class Key>
__device__ __forceinline__ void choose(const Key& key, int tiles, int nk, int lead, int n, bool all, int words, uint64_t* out) {
  const int lane = threadIdx.x % kWave;
  // Which of a tile's blocks compete: those past the leading ones.
  auto rest = [&](int t) {
    const int lo = std::min(64, std::max(0, lead - 64 * t)), up = std::min(64, std::max(0, nk - 64 * t));
    const uint64_t below = up == 64 ? ~uint64_t(0) : (uint64_t(1) << up) - 1;
    return lo == 64 ? 0 : below & (~uint64_t(0) << lo);
  };
  // The largest threshold that n keys reach, bit by bit; `exact`: just n do.
  uint64_t top = 0;
  bool exact = all || n == 0 || n == nk - lead;
  for (int bit = 63; bit >= 0 && !exact; --bit) {
    const uint64_t cand = top | (uint64_t(1) << bit);
    int count = 0;
    _Pragma("unroll(HELD ? HELD : 1)") for (int t = 0; t < (HELD ? HELD : tiles); ++t) count += __popcll(__ballot(key(t) >= cand));
    if (count >= n) top = cand;
    exact = count == n;
  }
  int spare = 0;  // how many of the keys equal to the threshold count
  if (!exact) {
    int above = 0;
    _Pragma("unroll(HELD ? HELD : 1)") for (int t = 0; t < (HELD ? HELD : tiles); ++t) above += __popcll(__ballot(key(t) > top));
    spare = n - above;
  }
  _Pragma("unroll(HELD ? HELD : 1)") for (int t = 0; t < (HELD ? HELD : tiles); ++t) {
    if (t >= tiles) continue;
    const uint64_t in = rest(t), k = key(t);
    const uint64_t past = nk - 64 * t >= 64 ? ~uint64_t(0) : (uint64_t(1) << (nk - 64 * t)) - 1;
    uint64_t on = past & ~in;  // the leading ones
    if (all) on = past;
    else if (n > 0) on |= __ballot(exact ? k >= top : k > top) & in;
    if (!exact) {
      const uint64_t tie = __ballot(k == top) & in;
      const int before = __popcll(tie & ((uint64_t(1) << lane) - 1));
      on |= __ballot((tie >> lane & 1) && before < spare);
      spare -= std::min(spare, int(__popcll(tie)));
    }
    if (lane == 0) out[t] = on;
  }
  for (int w = tiles + lane; w < words; w += kWave) out[w] = 0;
}

template <int D>
__global__ __launch_bounds__(64 * kSelWaves) void block_select_kernel(const SelectArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint64_t keys[];
  // Heads vary fastest over the workgroups: a head's stay on one XCD (for multiples of eight), whose L2 then reads its
  // keys' means once.
  const unsigned wg = unsigned(wide_block());
  const int h = int(wg % unsigned(a.H)), group = int(wg / unsigned(a.H)), hk = h / (a.H / a.Hk), lane = threadIdx.x % kWave, l16 = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (group >= a.groups[kMaxSeqs]) return;
  int q_blk = a.seq.q_blk[0], q_end = a.seq.q_blk[1], k_blk = a.seq.k_blk[0], nk = a.seq.k_blk[1] - k_blk, g0 = 0;
#pragma unroll
  for (int b = 1; b < kMaxSeqs; ++b)
    if (b < a.seq.B && group >= a.groups[b])
      q_blk = a.seq.q_blk[b], q_end = a.seq.q_blk[b + 1], k_blk = a.seq.k_blk[b], nk = a.seq.k_blk[b + 1] - k_blk, g0 = a.groups[b];
  const int i0 = (group - g0) * a.rows;  // the workgroup's first query block of its sequence
  const int n_rows = std::min(a.rows, q_end - q_blk - i0);
  const int lead = std::min(nk, (a.k_lead + kKB - 1) / kKB);
  // 16 rows in product order (lane l: row l % 16, of each eight elements those at 2 (l / 16)), fetched a
  // quarter (or half) row to 16 lanes, 16-byte chunk c of row r through LDS at c ^ r.
  char* mine = reinterpret_cast<char*>(keys) + wave * 4096;
  auto rows16 = [&](const double* base, int64_t ld, int last, f64x2(&f)[D / 8]) __attribute__((always_inline)) {
    f64x2 raw[D / 8];
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        raw[4 * c + i] = *reinterpret_cast<const f64x2*>(base + std::min(4 * i + g, last) * ld + 32 * c + 2 * l16);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<f64x2*>(mine + (4 * i + g) * 256 + ((l16 ^ (4 * i + g)) * 16)) = raw[4 * c + i];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[4 * c + i] = *reinterpret_cast<const f64x2*>(mine + l16 * 256 + (((4 * i + g) ^ l16) * 16));
    }
  };
  uint64_t* scores = keys + kSelWaves * 512;  // [rows][nk]
  f64x2 q[D / 8];
  if (16 * wave < nk) rows16(a.qm + (int64_t(q_blk + i0) * a.H + h) * D, int64_t(a.H) * D, n_rows - 1, q);
  for (int t = wave; 16 * t < nk; t += kSelWaves) {
    f64x2 k[D / 8];
    rows16(a.km + (int64_t(k_blk + 16 * t) * a.Hk + hk) * D, int64_t(a.Hk) * D, nk - 16 * t - 1, k);
    f64x4 acc = {0.0, 0.0, 0.0, 0.0}, odd = acc;
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      acc = __builtin_amdgcn_mfma_f64_16x16x4f64(q[c].x, k[c].x, acc, 0, 0, 0);
      odd = __builtin_amdgcn_mfma_f64_16x16x4f64(q[c].y, k[c].y, odd, 0, 0, 0);
    }
    // Register r holds row 4 r + lane / 16 of column lane % 16.
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 4 * r + g;
      if (row < n_rows && 16 * t + l16 < nk) scores[int64_t(row) * nk + 16 * t + l16] = order_key(acc[r] + odd[r]);
    }
  }
  __syncthreads();
  const int tiles = (nk + 63) / 64, n = std::min(a.keep, nk - lead);
  for (int r = wave; r < n_rows; r += kSelWaves) {
    const int i = i0 + r;
    const bool all = int64_t(i) * kQB < a.q_lead;
    const uint64_t* row = scores + int64_t(r) * nk;
    uint64_t* out = a.mask + (int64_t(h) * a.seq.q_blk[kMaxSeqs] + q_blk + i) * a.words;
    auto at = [&](int t) { return 64 * t + lane < nk && 64 * t + lane >= lead ? row[64 * t + lane] : 0; };
    auto held = [&](auto tag) {
      constexpr int T = decltype(tag)::value;
      uint64_t k[T];
#pragma unroll
      for (int t = 0; t < T; ++t) k[t] = at(t);
      choose<T>([&](int t) { return k[t]; }, tiles, nk, lead, n, all, int(a.words), out);
    };
    if (tiles <= 1) held(std::integral_constant<int, 1>());
    else if (tiles <= 2) held(std::integral_constant<int, 2>());
    else if (tiles <= 4) held(std::integral_constant<int, 4>());
    else if (tiles <= 8) held(std::integral_constant<int, 8>());
    else choose<0>(at, tiles, nk, lead, n, all, int(a.words), out);
  }
}

}  // namespace
}  // namespace avits

using namespace avits;

extern "C" int avits_block_means(const void* x, int64_t ld, int64_t M, int32_t H, int32_t d, int32_t block, int32_t B,
                                 const int64_t* off, int dtype, double* means, void* stream) {
  MeanArgs a{};
  const int rc = seq_rows("block_means", B, off, M, block == kQB ? kQB : kKB, a.row, a.blk);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(block == kQB || block == kKB, "block_means: block=%d (need %d or %d)", block, kQB, kKB);
  AVITS_REQUIRE(H >= 1 && H <= 1024, "block_means: H=%d outside [1, 1024]", H);
  if (d != 64 && d != 128) return set_error(AVITS_ERR_UNSUPPORTED, "block_means: head dim %d (need 64 or 128)", d);
  if (dtype != AVITS_F32 && dtype != AVITS_BF16) return set_error(AVITS_ERR_UNSUPPORTED, "block_means: dtype %d unsupported", dtype);
  const int64_t cols = int64_t(H) * d, elem = dtype == AVITS_BF16 ? 2 : 4;
  const int n = a.blk[B];
  if (n == 0) return AVITS_OK;
  AVITS_REQUIRE(x && means, "block_means: null pointer");
  AVITS_REQUIRE((M <= 1 || ld >= cols) && ld < (int64_t(1) << 31) && ld * elem % 16 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(means) % 16 == 0,
                "block_means: rows at least H * d apart and on 16 bytes (row stride %lld)", (long long)ld);
  a.x = x;
  a.ld = ld;
  a.out = means;
  a.B = B;
  a.block = block;
  a.blocks = n;
  a.cols = int(cols);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  TimedLaunch timed("block_means", s);
  const int per = 32 * int(16 / elem);
  const dim3 grid = wide_grid(n, static_cast<unsigned>((cols + per - 1) / per));
  if (dtype == AVITS_BF16) hipLaunchKernelGGL((block_means_kernel<bf16_t>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((block_means_kernel<float>), grid, dim3(256), 0, s, a);
  return launch_status("block_means");
}

extern "C" int avits_block_select(const double* q_means, const double* k_means, int64_t M, int64_t N, int32_t B, const int64_t* q_off,
                                  const int64_t* k_off, int32_t H, int32_t Hk, int32_t d, int64_t q_lead, int64_t k_lead, int64_t keep,
                                  uint64_t* mask, int64_t words, void* stream) {
  SelectArgs a{};
  const int rc = seq_blocks(a.seq, "block_select", B, q_off, M, k_off, N);
  if (rc != AVITS_OK) return rc;
  AVITS_REQUIRE(Hk >= 1 && H >= Hk && H % Hk == 0 && H <= 1024, "block_select: H=%d must be a multiple of Hk=%d, at most 1024", H, Hk);
  if (d != 64 && d != 128) return set_error(AVITS_ERR_UNSUPPORTED, "block_select: head dim %d (need 64 or 128)", d);
  AVITS_REQUIRE(q_lead >= 0 && k_lead >= 0 && keep >= 0, "block_select: q_lead, k_lead and keep must be >= 0");
  int nk = 0;
  for (int b = 0; b < B; ++b) nk = std::max(nk, a.seq.k_blk[b + 1] - a.seq.k_blk[b]);
  if (nk > kMaxKeyBlocks)
    return set_error(AVITS_ERR_UNSUPPORTED, "block_select: a sequence of %d key blocks (at most %d)", nk, kMaxKeyBlocks);
  AVITS_REQUIRE(words >= (nk + 63) / 64 && words < (int64_t(1) << 20), "block_select: %lld words a row for %d key blocks", (long long)words, nk);
  const int nq = a.seq.q_blk[B];
  if (nq == 0 || words == 0) return AVITS_OK;
  AVITS_REQUIRE(q_means && mask && (k_means || a.seq.k_blk[B] == 0), "block_select: null pointer");
  AVITS_REQUIRE(reinterpret_cast<uintptr_t>(q_means) % 16 == 0 && reinterpret_cast<uintptr_t>(k_means) % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(mask) % 8 == 0,
                "block_select: misaligned pointer");
  a.qm = q_means;
  a.km = k_means;
  a.mask = mask;
  a.words = words;
  a.H = H, a.Hk = Hk, a.d = d;
  const int64_t most = (int64_t(1) << 31) - 1 - 4096;
  a.q_lead = int(std::min(q_lead, most));
  a.k_lead = int(std::min(k_lead, most));
  a.keep = int(std::min(keep, most));
  // As many query blocks to a workgroup as a product has rows, fewer where their scores would not fit.
  a.rows = std::max(1, std::min(16, kMaxKeyBlocks / std::max(nk, 1)));
  for (int b = 0; b < B; ++b) a.groups[b + 1] = a.groups[b] + (a.seq.q_blk[b + 1] - a.seq.q_blk[b] + a.rows - 1) / a.rows;
  a.groups[kMaxSeqs] = a.groups[B];
  if (int64_t(a.groups[B]) * H >= int64_t(1) << 31)
    return set_error(AVITS_ERR_UNSUPPORTED, "block_select: %d query blocks of %d heads", nq, H);
  a.seq.q_blk[kMaxSeqs] = nq;
  const size_t lds = size_t(a.rows) * nk * sizeof(uint64_t) + kSelWaves * 4096;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const auto kernel = d == 128 ? &block_select_kernel<128> : &block_select_kernel<64>;
  if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                             kMaxKeyBlocks * int(sizeof(uint64_t)) + kSelWaves * 4096) != hipSuccess)
    return set_error(AVITS_ERR_HIP, "block_select: no %zu bytes of LDS", lds);
  TimedLaunch timed("block_select", s);
  hipLaunchKernelGGL(kernel, wide_grid(int64_t(a.groups[B]) * H), dim3(64 * kSelWaves), lds, s, a);
  return launch_status("block_select");
}
