// How the owners of query (key) blocks share their lists, whose lengths only the mask knows.
//
// A unit is a block of a head; its list is the blocks that it walks.  A list longer than T = a
// 512th of all lists together (two shares to a CU), and at least kMinList, is cut into pieces of at most T that run as workgroups of their
// own; their sums go to slots, and a second kernel joins them in order.  There are at most 512 such
// lists and 1024 pieces.  Pieces run first, then the longer of the uncut lists: a long list (a block
// of text rows keeps everything) that one workgroup walked would go on when the chip is done with the rest.
// More than kMaxUnits, a round and a half of the 512 workgroups, even out by themselves.  With text of a sixteenth
// of the blocks and a quarter of the rest kept: 4600 rows of 8 heads of 128 (288 units) 73 us, without a plan 88; 5171 rows
// of 16 heads of 64 (656 units), forward kernels 50 and 58; 8200 rows of 16 heads of 128 (1040 units) 226 and 206; dk and dv
// at 1152 units of 128, 10 us of 290 slower with one.
#pragma once

#include "sparse_attn.h"

namespace avits {

constexpr int kMaxUnits = 768, kShares = 512, kMaxSlots = 2 * kShares, kMinList = 8;

// One side's plan in memory: n_items, n_cut, then kMaxSlots + units items (unit, piece | pieces << 16, list's length, first slot), then
// the cut lists (unit, pieces, first slot).
struct SparsePlan {
  int4 head;
  int4 items[kMaxSlots + kMaxUnits];
  int4 cut[kShares];
};

// Run by one workgroup of NT threads.  KEYS: the units are key blocks of key heads.
template <bool KEYS, int NT>
__device__ void sparse_plan(const SparseArgs& a, SparsePlan* plan, int* counts, uint64_t* sums) {
  const int tid = threadIdx.x, nq = a.seq.q_blk[kMaxSeqs], Hk = a.H / a.group;
  const int units = KEYS ? a.seq.k_blk[kMaxSeqs] * Hk : nq * a.H;
  if constexpr (KEYS) {
    for (int u = tid; u < units; u += NT) counts[u] = 0;
    __syncthreads();
  }
  for (int e = tid; e < nq * a.H; e += NT) {  // a query block of a head: its words
    const int blk = e / a.H, h = e % a.H;
    const Seq s = seq_of<false>(a.seq, blk);
    const uint64_t* row = a.mask ? a.mask + (int64_t(h) * nq + blk) * a.words : nullptr;
    int n = 0;
    for (int w = 0; 64 * w < s.nk; ++w) {
      uint64_t on = row ? row[w] : ~uint64_t(0);
      if (s.nk - 64 * w < 64) on &= (uint64_t(1) << (s.nk - 64 * w)) - 1;
      if constexpr (KEYS) {
        for (; on != 0; on &= on - 1) atomicAdd(&counts[(s.kb + 64 * w + __builtin_ctzll(on)) * Hk + h / a.group], 1);
      } else {
        n += __popcll(on);
      }
    }
    if constexpr (!KEYS) counts[e] = n;
  }
  __syncthreads();
  // All lists together, and the longest piece.
  int mine = 0;
  for (int u = tid; u < units; u += NT) mine += counts[u];
  sums[tid] = mine;
  __syncthreads();
  for (int o = NT / 2; o > 0; o /= 2) {
    if (tid < o) sums[tid] += sums[tid + o];
    __syncthreads();
  }
  const int most = std::max(kMinList, int((sums[0] + kShares - 1) / kShares));
  __syncthreads();
  // Places by a running sum of (pieces, cut lists, long lists, short lists), 16 bits each: a thread has
  // consecutive units.
  const int per = (units + NT - 1) / NT, lo = std::min(units, tid * per), up = std::min(units, lo + per);
  auto weigh = [&](int n) {
    if (n > most) return uint64_t((n + most - 1) / most) | uint64_t(1) << 16;
    return uint64_t(1) << (2 * n > most ? 32 : 48);
  };
  uint64_t own = 0;
  for (int u = lo; u < up; ++u) own += weigh(counts[u]);
  sums[tid] = own;
  __syncthreads();
  for (int o = 1; o < NT; o *= 2) {
    const uint64_t v = tid >= o ? sums[tid - o] : 0;
    __syncthreads();
    sums[tid] += v;
    __syncthreads();
  }
  const uint64_t all = sums[NT - 1];
  uint64_t at = sums[tid] - own;
  const int pieces_all = int(all & 0xffff), long_all = int(all >> 32 & 0xffff);
  for (int u = lo; u < up; ++u) {
    const uint64_t w = weigh(counts[u]);
    if (w & 0xffff) {
      const int first = int(at & 0xffff), pieces = int(w & 0xffff);
      for (int p = 0; p < pieces; ++p) plan->items[first + p] = make_int4(u, p | pieces << 16, counts[u], first);
      plan->cut[at >> 16 & 0xffff] = make_int4(u, pieces, first, 0);
    } else {
      const int place = w >> 32 & 0xffff ? int(at >> 32 & 0xffff) : long_all + int(at >> 48);
      plan->items[pieces_all + place] = make_int4(u, 1 << 16, counts[u], 0);
    }
    at += w;
  }
  if (tid == 0) plan->head = make_int4(pieces_all + long_all + int(all >> 48), int(all >> 16 & 0xffff), 0, 0);
}

// The work of workgroup b: unit, piece | pieces << 16, the list's length (from a plan) and first slot; unit -1: none.
__device__ __forceinline__ int4 sparse_item(const SparseArgs& a, int units, int b) {
  if (!a.plan) return make_int4(b % units, b / units | a.pieces << 16, 0, b % units);
  if (b >= a.plan->head.x) return make_int4(-1, 1 << 16, 0, 0);
  return a.plan->items[b];
}
// The slot of a piece.
__device__ __forceinline__ int64_t sparse_slot(const SparseArgs& a, int units, int first, int piece) {
  return a.plan ? first + piece : first + int64_t(piece) * units;
}
// The cut list that workgroup b / per of a joining kernel works on: unit, pieces, first slot; unit -1: none.
__device__ __forceinline__ int4 sparse_cut(const SparseArgs& a, int b) {
  if (!a.plan) return make_int4(b, a.pieces, b, 0);
  if (b >= a.plan->head.y) return make_int4(-1, 0, 0, 0);
  return a.plan->cut[b];
}

// Host: slots that a side can need.
inline int64_t sparse_slots(int64_t units, int64_t most_list) {
  return std::min<int64_t>(kMaxSlots, units * ceil_div64(most_list, kMinList));
}

}  // namespace avits
