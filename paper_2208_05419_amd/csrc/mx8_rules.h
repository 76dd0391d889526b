// mx8_rules.h -- which kernel a product of rows in eight bits takes, how it is cut, and its workspace: rules on sizes.
// Host code without HIP, so that a test can compile it and walk over them.
#pragma once
#include "linear_rules.h"

namespace afno {

// ld: bytes of a row, K rounded up to 32.  Times with GELU, M x 1,024 x 1,024 unless said, the join of the splits among them.
// bf16, 256: a CU has one workgroup of it and two of 128, so it pays from where those take a second round, more than 512
// tiles of 128 (576 of them, 9,216 rows: 27.7 us, 128 29.6; of 256 k's 18.2 and 19.3, of 4,096 61.4 and 73.9; but 512: 27.2 and
// 21.7), but for a second round of its own that is a third full (275 tiles, 17,600 rows: 50.8 and 46.4, of 128 k's 31.6 and
// 22.7; 350 tiles: 52.2 and 52.6; 512: 55.6 and 69.1).  The epilogue and the columns behind a narrow N are not
// asked for.  64,800 x 1,024 x 4,096 with GELU in eight bits 409 and (128) 462; with dropout and the value before in eight
// bits, too, 595 and 555, with dropout and a residual 686 and 649, 12,960 rows 146 and 119, 147 and 122: there 128 is
// ahead, one workgroup's epilogue beside the other's products; of 4,096 k's it is not (64,800 x 4,096 x 1,024 309 and 393,
// 318 and 408).
// 64,800 x 1,024 x 264 58.4 and 52.8, x 320 55.8 and 51.9; x 64 in tiles of 128 20.4, of 64 21.5, x 8 19.5 and 19.3.
// 128 where three in four CUs get a tile (200 tiles: 14.2, 64 17.4; 128 tiles: 13.8 and 10.4), in fp32 but for a few more
// than the CUs (fp32: 200 tiles 19.9 and 21.5, 256 21.1 and 22.8, 320 29.5 and 27.5, 400 30.7 and 35.0, 4,096 222 and 297).
// Splits of k where tiles of 64 leave CUs without one, of 1,024 k's at least (64 x 4,096 x 1,024, 16 tiles: 9.7 us in
// four, 11.6 whole, fp32 11.3 in four, 13.8 in two, 18.3 whole; 128 x 4,096 x 4,096, 128 tiles: 13.7 in two, 14.3 whole;
// 64 x 1,024 x 4,096 8.7 in two of 512, 6.3 whole).
inline Cut cut_mx8(int64_t M, int64_t N, int64_t ld, int es) {
  Cut c;
  auto tiles = [&](int t) { return ceil_div(M, t) * ceil_div(N, t); };
  auto cut = [&](int tile, int64_t s) {
    c.tile = tile;
    c.kper = std::max<int64_t>(128, ceil_div(ceil_div(ld, s), 128) * 128);
    c.splits = (int)ceil_div(ld, c.kper);
    return c;
  };
  const int64_t t256 = tiles(256), t128 = tiles(128);
  if (es == 2 && t128 > 512 && (t256 <= 256 || t256 >= 340)) return cut(256, 1);
  if (t128 >= 192 && (es == 2 || t128 <= 256 || t128 >= 360)) return cut(128, 1);
  const int64_t t = tiles(64);
  return cut(64, t >= 256 ? 1 : std::max<int64_t>(1, std::min<int64_t>(256 / t, ld / 1024)));
}
// Whether mx8_rows takes the product (with GELU in a graph of twenty such calls, bf16: 1,024 x 4,096 4.2 us for one row, 4.7 for
// sixteen, where mx8_gemm_tile takes 5.5 and 5.6; 2,048 x 512 5.4 and 7.3, sixteen rows 6.5 and 7.4; 2,048 x 4,096,
// sixteen rows, 6.7 and 7.5; fp32 4.4 and 7.3, 5.0 and 7.4 at 1,024 x 4,096.  More k's would be a second stage of each wave:
// 4,096 x 1,024, sixteen rows, 10.6 with one, 8.9 in tiles).
constexpr int kFewRowsWaves = 16;  // a workgroup's, a stage of 128 k's each
inline bool mx8_few_rows(int64_t M, int64_t ld) { return M <= 16 && ld <= 128 * kFewRowsWaves; }
inline size_t mx8_part_bytes(int64_t M, int64_t N, int64_t ld, int es) {
  return mx8_few_rows(M, ld) ? 0 : part_of(M, N, cut_mx8(M, N, ld, es));
}

// The scales that mx8_gemm_tile256 has in the LDS: of each of its 512 rows 16 bytes, in one of two buffers for stages `first`
// .. first + 3 (first a multiple of four).  Rows of `blocks` scales; 16 of them at least from the fourth stage on.
constexpr int kScaleRows256 = 512;
// the row's block in the first of the 16 bytes of the stages behind `first` .. + 3: theirs, or what leaves the load within the
// row (of stages 0 .. 3: block 0)
constexpr int next_scales256(int first, int blocks) { return std::min(4 * first + 16, blocks - 16); }
// where the first block of stage first + j is, from the buffers' begin on; rows are 16 bytes apart
constexpr int scales_at256(int first, int j, int blocks) {
  const int shift = first ? 4 * first - std::min(4 * first, blocks - 16) : 0;
  return 16 * kScaleRows256 * (first >> 2 & 1) + shift + 4 * j;
}
// how far ahead of block gq lane group gq reads where `there` of a stage's four are there: the last one for those behind it,
// whose own place would be in the next row, or behind the array
constexpr int scale_back256(int gq, int there) { return gq < there ? 0 : gq - (there - 1); }

}  // namespace afno
