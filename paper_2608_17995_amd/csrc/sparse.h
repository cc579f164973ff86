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

// Host: checks the offsets (null: one sequence of all rows) and cuts the blocks.
int seq_blocks(SeqBlocks& s, const char* what, int32_t B, const int64_t* q_off, int64_t M, const int64_t* k_off, int64_t N);
int seq_rows(const char* what, int32_t B, const int64_t* off, int64_t rows, int block, int32_t* row, int32_t* blk);

}  // namespace avits
