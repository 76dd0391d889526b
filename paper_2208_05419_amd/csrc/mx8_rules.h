// mx8_rules.h -- which kernel a product of rows in eight bits takes, how it is cut, and its workspace: rules on sizes.
// Host code without HIP, so that a test can compile it and walk over them.
#pragma once
#include "linear_rules.h"

namespace afno {

// ld: bytes of a row, K rounded up to 32.  Times with GELU, the join of the splits among them.
// bf16: 256 where some five CUs in eight get a tile of it (9,600 x 1,024 x 1,280, 190 tiles: 28.5 us, 128 35.0; 4,096 x
// 1,024 x 4,096, 256 tiles: 35.6, 128 42.8; but 4,096 x 1,024 x 2,048, 128 tiles: 26.4 and 23.0, 6,400 x 4,096 x 1,024, 100
// tiles: 58.1 and 44.9), 128 where three in four get one (10,368 x 1,536 x 384, 243 tiles: 17.9, 64 20.4; 2,100 x 4,096 x
// 1,024, 136 tiles: 32.7 and 31.5).  fp32: 64, whose four workgroups a CU cover each other's conversions (64,800 x
// 1,024 x 1,024: 279 us, 128 362; 10,368 x 384 x 1,536 46 and 95; of longer rows, 16,200 x 4,096 x 1,024, 198 and 177).
// Splits of k where tiles of 64 leave CUs without one, of 1,024 k's at least (64 x 4,096 x 1,024, 16 tiles: 9.7 us in
// four, 11.6 whole, fp32 13.8 in two and 18.5; 128 x 4,096 x 4,096, 128 tiles: 13.7 in two, 14.3 whole; 64 x
// 1,024 x 4,096 8.7 in two of 512, 6.3 whole).
inline Cut cut_mx8(int64_t M, int64_t N, int64_t ld, int es) {
  Cut c;
  auto tiles = [&](int t) { return ceil_div(M, t) * ceil_div(N, t); };
  auto cut = [&](int tile, int64_t s) {
    c.tile = tile;
    c.kper = std::max<int64_t>(128, ceil_div(ceil_div(ld, s), 128) * 128);
    c.splits = (int)ceil_div(ld, c.kper);
    return c;
  };
  if (es == 2 && tiles(256) >= 160) return cut(256, 1);
  if (es == 2 && tiles(128) >= 192) return cut(128, 1);
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
