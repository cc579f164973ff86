// Sequences packed one after another, cut into query blocks of 128 rows and key
// blocks of 64, and the words that say which key blocks a query block attends to.
#pragma once

#include "kernels.h"

namespace avits {

constexpr int kQB = AVITS_Q_BLOCK, kKB = AVITS_K_BLOCK;

// Sequence b's query rows [q_row[b], q_row[b + 1]) and query blocks
// [q_blk[b], q_blk[b + 1]), its key rows and key blocks.
struct SeqBlocks {
  int32_t B;
  int32_t q_row[kMaxSeqs + 1], k_row[kMaxSeqs + 1], q_blk[kMaxSeqs + 1], k_blk[kMaxSeqs + 1];
};

// One sequence's share of the above.
struct Seq {
  int q_lo, q_hi, k_lo, k_hi;  // rows
  int qb, kb, nk;              // first blocks, key blocks
};

// The sequence that query (key) block `blk` belongs to: unrolled, so that no
// index into the arguments is dynamic (that would copy them to private memory).
template <bool KEYS>
__device__ __forceinline__ Seq seq_of(const SeqBlocks& a, int blk) {
  Seq s{a.q_row[0], a.q_row[1], a.k_row[0], a.k_row[1], a.q_blk[0], a.k_blk[0], a.k_blk[1] - a.k_blk[0]};
#pragma unroll
  for (int b = 1; b < kMaxSeqs; ++b)
    if (b < a.B && blk >= (KEYS ? a.k_blk[b] : a.q_blk[b]))
      s = Seq{a.q_row[b], a.q_row[b + 1], a.k_row[b], a.k_row[b + 1], a.q_blk[b], a.k_blk[b], a.k_blk[b + 1] - a.k_blk[b]};
  return s;
}

// A launch has fewer than 2^32 threads along x (it drops the rest without an error): n workgroups, in rows of 2^20 along
// y where they are more, the last row not whole.
inline dim3 wide_grid(int64_t n, unsigned z = 1) {
  const int64_t x = std::min<int64_t>(n, int64_t(1) << 20);
  return dim3(unsigned(x), unsigned(ceil_div64(n, std::max<int64_t>(x, 1))), z);
}
__device__ __forceinline__ int64_t wide_block() { return int64_t(blockIdx.y) * gridDim.x + blockIdx.x; }
// Whether n workgroups fit along x alone.
inline bool fits_x(int64_t n, int threads) { return n * threads < int64_t(1) << 32; }

// Host: checks the offsets (null: one sequence of all rows) and cuts the blocks.
int seq_blocks(SeqBlocks& s, const char* what, int32_t B, const int64_t* q_off, int64_t M, const int64_t* k_off, int64_t N);
int seq_rows(const char* what, int32_t B, const int64_t* off, int64_t rows, int block, int32_t* row, int32_t* blk);

}  // namespace avits
