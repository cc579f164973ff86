// Arguments of the sparse attention kernels and the walk over a query block's key blocks.
#pragma once

#include "sparse.h"

namespace avits {

struct SparseArgs {
  const void *q, *k, *v, *dout;
  void *o, *dq, *dk, *dv;
  int64_t q_ld, k_ld, v_ld, do_ld, o_ld, dq_ld, dk_ld, dv_ld;
  const uint64_t* mask;  // [H][query blocks][words], or null: every block
  int64_t words;
  float* lse;            // [H][M]
  float* delta;          // [H][M]: do . o
  int64_t M;
  int H, group, d;       // query heads, query heads to a key head
  float scale;
  SeqBlocks seq;         // q_row, q_blk: the totals also in their last entry
};

// The key blocks that query block blk of head h keeps, in order (wave-uniform).
struct BlockWalk {
  const uint64_t* row;
  int nk, w, total;
  uint64_t cur;
  __device__ __forceinline__ BlockWalk(const SparseArgs& a, int h, int blk, int n) {
    row = a.mask ? a.mask + (int64_t(h) * a.seq.q_blk[kMaxSeqs] + blk) * a.words : nullptr;
    nk = n;
    w = 0;
    total = 0;
    for (int i = 0; 64 * i < nk; ++i) total += __popcll(word(i));
    cur = nk > 0 ? word(0) : 0;
  }
  // Word i without the bits past the last key block.
  __device__ __forceinline__ uint64_t word(int i) const {
    const uint64_t all = nk - 64 * i >= 64 ? ~uint64_t(0) : (uint64_t(1) << (nk - 64 * i)) - 1;
    return row ? row[i] & all : all;
  }
  __device__ __forceinline__ int next() {
    while (cur == 0) {
      ++w;
      if (64 * w >= nk) return -1;
      cur = word(w);
    }
    const int j = 64 * w + __builtin_ctzll(cur);
    cur &= cur - 1;
    return j;
  }
};

// Whether query block blk of head h keeps its sequence's key block j.
__device__ __forceinline__ bool kept(const SparseArgs& a, int h, int blk, int j) {
  return !a.mask || (a.mask[(int64_t(h) * a.seq.q_blk[kMaxSeqs] + blk) * a.words + j / 64] >> (j % 64) & 1);
}

}  // namespace avits
