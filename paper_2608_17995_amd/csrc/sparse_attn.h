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
  float2* stats;         // [H][M]: lse and do . o, for the backward pass
  int64_t M;
  int H, group, d;       // query heads, query heads to a key head
  float scale;
  const struct SparsePlan* plan;  // which lists are cut, by the mask; or null:
  int64_t slots;         // with a plan: its slots
  int pieces;            // of each unit's list, joined afterwards (1: none)
  float* part;           // slots of unfinished sums: [128][d] of outputs or dq, or [2][64][d] of dk and dv
  float* part_ml;        // slots of [128] (maximum in the log2 domain, sum)
  SeqBlocks seq;         // q_row, q_blk, k_blk: the totals also in their last entry
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
  __device__ __forceinline__ void skip(int n) {
    if (n == 0) return;
    while (n >= int(__popcll(cur))) {
      n -= __popcll(cur);
      cur = 0;
      ++w;
      if (64 * w >= nk) return;
      cur = word(w);
    }
    for (; n > 0; --n) cur &= cur - 1;
  }
};

// The forward pass's pieces of every list where there are few units: two workgroups to each of 256 CUs, each with two blocks at
// least where the mask keeps everything.  (What it keeps is not known here: pieces of a list of few blocks may have none.)
constexpr int kMaxPieces = 64, kFewUnits = 64;
inline int sparse_pieces(int64_t units, int64_t most_list) {
  if (units > kFewUnits || units == 0) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / units, most_list / 2), kMaxPieces)));
}
void launch_sparse_bf16(const SparseArgs& a, hipStream_t s);
void launch_sparse_back_bf16(const SparseArgs& q, const SparseArgs& k, hipStream_t s);  // one plan for each

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

// Transposing read: of 16 lanes, lane i gives the address of four 16-bit elements of row i / 4,
// columns 4 (i % 4) .., and receives column i of the four rows.
__device__ __forceinline__ u32x2 lds_read_tr(const char* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
}

// The factor of a sequence's sums for dq and dk.  Over one key the probability is 1 whatever q and k are, so these
// are zero: the sums hold what dout . v and dout . o differ by in the order of their additions.
__device__ __forceinline__ float grad_scale(const SparseArgs& a, const Seq& s) { return s.k_hi - s.k_lo == 1 ? 0.f : a.scale; }

// Whether query block blk of head h keeps its sequence's key block j.
__device__ __forceinline__ bool kept(const SparseArgs& a, int h, int blk, int j) {
  return !a.mask || (a.mask[(int64_t(h) * a.seq.q_blk[kMaxSeqs] + blk) * a.words + j / 64] >> (j % 64) & 1);
}

}  // namespace avits
