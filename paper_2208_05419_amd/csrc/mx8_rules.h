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
// Whether mx8_rows takes the product (with GELU, bf16: 1,024 x 4,096 4.4 us for one row, 4.9 for sixteen, where mx8_gemm_tile
// takes 5.8 for either; 2,048 x 512, sixteen rows 6.8 and 7.8; but 4,096 x 1,024 10.6 and 8.9, one row 8.4 and 8.2).
inline bool mx8_few_rows(int64_t M, int64_t ld) { return M <= 16 && ld <= 2048; }
inline size_t mx8_part_bytes(int64_t M, int64_t N, int64_t ld, int es) {
  return mx8_few_rows(M, ld) ? 0 : part_of(M, N, cut_mx8(M, N, ld, es));
}

}  // namespace afno
