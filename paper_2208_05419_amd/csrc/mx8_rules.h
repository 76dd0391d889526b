// mx8_rules.h -- which kernel a product of rows in eight bits takes, how it is cut, and its workspace: rules on sizes.
// Host code without HIP, so that a test can compile it and walk over them.
#pragma once
#include "linear_rules.h"

namespace afno {

// ld: bytes of a row, K rounded up to 32
inline Cut cut_mx8(int64_t M, int64_t N, int64_t ld, int es) {
  Cut c;
  if (es == 2 && ceil_div(M, 256) * ceil_div(N, 256) >= 128) return {256, 1, ceil_div(ld, 128) * 128};
  auto tiles = [&](int t) { return ceil_div(M, t) * ceil_div(N, t); };
  auto cut = [&](int tile, int64_t s) {
    c.tile = tile;
    c.kper = std::max<int64_t>(128, ceil_div(ceil_div(ld, s), 128) * 128);
    c.splits = (int)ceil_div(ld, c.kper);
    return c;
  };
  if (tiles(128) >= 256) return cut(128, 1);
  const int64_t t = tiles(64);
  return cut(64, t >= 256 ? 1 : std::max<int64_t>(1, std::min<int64_t>(256 / t, ld / 1024)));
}
inline size_t mx8_part_bytes(int64_t M, int64_t N, int64_t ld, int es) {
  return part_of(M, N, cut_mx8(M, N, ld, es));
}

}  // namespace afno
