// Which output tile a workgroup of a matrix product takes.
#pragma once

#include <algorithm>

#include "common.h"

namespace avits {
namespace {

// Tile order of the ping-pong kernels, in 32-bit arithmetic (the 64-bit
// divisions of the general mapping cost about 1 us at the head of every
// workgroup).  Tiles of problem 0 come first.  A problem's row tiles form
// near-equal bands of at most kBand; a band's tiles walk down its rows, then
// over the columns, so the 32 tiles that run on one XCD together share about
// kBand row tiles and 4 weight tiles in its L2 (walking down all the rows
// of a long problem re-read A once per column of tiles).
constexpr uint32_t kBand = 8;
__device__ __forceinline__ void pp_place(uint32_t id, uint32_t tn, uint32_t tm0, uint32_t tm1, int& prob, int& row,
                                         int& col) {
  prob = id >= tn * tm0;
  const uint32_t local = prob ? id - tn * tm0 : id, tm = prob ? tm1 : tm0;
  const uint32_t bands = (tm + kBand - 1) / kBand, small = tm / bands, big = tm % bands;  // `big` bands of small + 1
  const uint32_t in_big = big * (small + 1) * tn;
  const bool first = local < in_big;
  const uint32_t rows = first ? small + 1 : small, u = first ? local : local - in_big;
  const uint32_t band = u / (rows * tn), v = u % (rows * tn);
  row = int((first ? 0 : big * (small + 1)) + band * rows + v % rows);
  col = int(v / rows);
}
__device__ __forceinline__ uint32_t xcd_logical_id32(uint32_t bid, uint32_t grid) {
  const uint32_t per = grid / 8, rem = grid % 8, x = bid % 8, i = bid / 8;
  return x * per + std::min(x, rem) + i;
}

}  // namespace
}  // namespace avits
