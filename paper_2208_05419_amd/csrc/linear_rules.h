// linear_rules.h -- which kernel a linear product takes, how it is cut, and what workspace a call needs:
// rules on sizes, element size and alignment.  Host code without HIP, so that a test can compile it and
// walk over them.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace afno {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t whole_units(int64_t n, int es) { return ceil_div(n, 16 / es) * (16 / es); }

// How a product is cut: the kernel's square tile, and splits of k whose sums join_splits adds.
struct Cut {
  int tile;  // 256: gemm_tile256; 128 or 64: gemm_tile, or gemm_reg where the operands are no 16-byte units
  int splits;
  int64_t kper;
};

// units: the operands are what the direct-to-LDS kernels take.  Times of the present kernels, the join of the
// splits among them.
// bf16: 256 where most CUs get a tile of it, also by a split of k that leaves 2,048 to each (64,800 k's, 1,024
// x 4,096: 450 us in four splits of 256, 592 in two of 128; 1,080 x 1,536 x 768, 30 tiles: 21 against
// 9 with 64).  Both: 128 where every CU gets one (bf16, 10,368 x 1,536 x 384, 972 tiles: 21 us, 64 30; at 256
// tiles, 4,096 x 1,024 x 1,024, about even: 18.5, 64 16.2 to 17.3), in fp32 from three in four (10,368 x 384 x
// 1,536, 243 tiles: dw 108, 64 115; but forward and dx 114 and 116, 64 103), or by splits of long sums (bf16,
// 10,368 k's in 384 x 1,536: 31 us in eight of 128, 41 with 64 whole), in fp32 two to a CU where 2,048 k's are
// left to each (20,000 k's, 2,048 x 2,048: 1,248 us in two splits, 1,411 whole; but 10,368 k's in 384 x 1,536:
// 121 in seven, 144 in ten).
// Else 64, split where the tiles leave CUs without one and the sum is long: a split costs the join's launch,
// about 3 us, and a stage of k's 0.2 us, in fp32 0.7 (bf16, 256 x 1,024 x 4,096, 64 tiles: 16.7 us whole,
// 11.4 in four; 64 x 4,096 x 1,024: 6.7 whole, 8.4 in two; fp32 20.5 whole, 13.1 in four).
// Without units every k-stage waits for its loads: splits until there are two workgroups a CU.
inline Cut cut_product(int64_t M, int64_t N, int64_t K, int es, bool units) {
  Cut c;
  auto tiles = [&](int t) { return ceil_div(M, t) * ceil_div(N, t); };
  auto cut = [&](int tile, int64_t s) {
    const int stage = 128 / es;
    c.tile = tile;
    c.kper = std::max<int64_t>(stage, ceil_div(ceil_div(K, s), stage) * stage);
    c.splits = (int)ceil_div(K, c.kper);
    return c;
  };
  auto fill = [&](int64_t t, int64_t want, int64_t least) {  // splits for `want` workgroups
    return std::max<int64_t>(1, std::min<int64_t>(want / t, K / least));
  };
  if (!units) {
    const int tile = M > 64 && N > 64 && tiles(128) * std::max<int64_t>(1, K / 256) >= 256 ? 128 : 64;
    return cut(tile, tiles(tile) >= 256 ? 1 : fill(tiles(tile), 512, tile == 128 ? 256 : 128));
  }
  if (es == 2) {
    const int64_t s = tiles(256) >= 128 ? 1 : fill(tiles(256), 256, 2048);
    if (tiles(256) * s >= 128) return cut(256, s);
  }
  const int64_t t128 = tiles(128);
  if (K >= 8192 && M > 64 && N > 64 && t128 < 512) {
    const bool two = es == 4 && 512 / t128 >= 1 && K / (512 / t128) >= 2048;
    return cut(128, fill(t128, two ? 512 : 256, 1024));
  }
  if (t128 >= 256 || (es == 4 && t128 >= 192)) return cut(128, 1);
  return cut(64, tiles(64) >= 256 ? 1 : fill(tiles(64), 256, es == 2 ? 1024 : 256));
}
inline size_t part_of(int64_t M, int64_t N, const Cut& c) {
  return c.splits > 1 ? (size_t)c.splits * M * N * sizeof(float) : 0;
}
// Whether linear_rows takes a forward product.  bf16, 1,024 x 4,096: 3.9 us for one row, 4.5 for two, 6.0 for
// four, where gemm_tile takes 6.5 for any; fp32 5.2 for eight, 9 for sixteen against 12.
inline bool few_rows(int64_t M, int es) { return M <= (es == 2 ? 2 : 16); }
// whatever the addresses turn out to be
inline size_t part_bytes(int64_t M, int64_t N, int64_t K, int es) {
  return std::max(part_of(M, N, cut_product(M, N, K, es, false)), part_of(M, N, cut_product(M, N, K, es, true)));
}

// D [M][N] = sum over k < K: an operand's leading dimension, its rows that are there to be read (row-major
// operands, ar and br: k is not their fastest index), whether it begins at a 16-byte boundary.
struct Product {
  bool ar, br;
  int64_t M, N, K, lda, ldb, ma, nb;
  bool a16, b16;
};
// The kernel: linear_rows, or one of cut's tile, from 16-byte units (the direct-to-LDS kernels) or from
// operands at any address and stride (gemm_reg).
struct Path {
  bool rows, units;
  Cut cut;
};
inline Path product_path(const Product& p, int es) {
  const int ue = 16 / es;
  Path r = {};
  r.rows = !p.ar && p.br && few_rows(p.M, es);
  r.units = p.lda % ue == 0 && p.ldb % ue == 0 && p.a16 && p.b16 && (!p.ar || p.ma % ue == 0) &&
            (!p.br || p.nb % ue == 0);
  if (!r.rows) r.cut = cut_product(p.M, p.N, p.K, es, r.units);
  return r;
}

// Whether operands that are no 16-byte units are copied to rows that are, for the direct-to-LDS kernels: a
// launch and a pass over them, against loads through registers.  bf16: 2,001 x 1,001 x 999 20 us, not
// copied 46; 300 x 77 x 333 7.6 and 6.3, but its gradients, whose factor dz comes in such rows anyway, 20 and 26.
// fp32, whose matrix instructions take longer than the loads: 54 and 74, but 1,000 x 1,001 x 501 27 and
// 27, and 64,800 x 77 x 1,023 with few operations to a byte 242 and 215.
inline bool worth_packing(int64_t M, int64_t K, int64_t N, int es, bool backward) {
  const double work = (double)M * (double)K * (double)N;
  if (es == 2) return work >= (backward ? 1 << 22 : 1 << 26);
  return work >= 1 << 30 && std::min(K, N) >= 256;
}

// Chunks of rows of the column sums: as many as fill the chip eight times with 256-column workgroups, of at
// least eight rows, one to a thread (1,080 x 1,536: 11.3 us with 32, 8.1 with eight).
inline int64_t chunk_rows(int64_t M, int64_t N) {
  const int64_t want = std::max<int64_t>(1, 2048 / ceil_div(N, 256));
  return std::max<int64_t>(8, ceil_div(ceil_div(M, want), 8) * 8);
}

// A linear call: x [M][K], w [K][N], which arrays begin at a 16-byte boundary, and, of a backward call, which
// gradients are asked for and whether an activation or dropout stands between g and dz.
struct LinearSizes {
  int64_t M, K, N;
  int es;
  bool x16, w16, g16, dx, dw, db, factor;
};
// Its workspace: copies of operands that are no 16-byte units (whatever the addresses turn out to be,
// room for them where the sizes are worth it), the factor dz, chunk sums, the splits' sums.
struct Layout {
  bool copy_x, copy_w, need_dz;
  int64_t kp, np;  // rows of the copies and of dz
  size_t x, w, dz, sums, part, bytes;
};
inline Layout forward_layout(const LinearSizes& a) {
  Layout l = {};
  if (few_rows(a.M, a.es)) return l;
  const bool packing = worth_packing(a.M, a.K, a.N, a.es, false);
  l.kp = whole_units(a.K, a.es);
  l.np = whole_units(a.N, a.es);
  l.copy_x = packing && (l.kp != a.K || !a.x16);
  l.copy_w = packing && (l.np != a.N || !a.w16);
  l.w = l.copy_x ? up256((size_t)a.M * l.kp * a.es) : 0;
  l.part = l.w + (l.copy_w ? up256((size_t)a.K * l.np * a.es) : 0);
  l.bytes = l.part + part_bytes(a.M, a.N, a.K, a.es);
  return l;
}
inline Layout backward_layout(const LinearSizes& a) {
  Layout l = {};
  const bool packing = worth_packing(a.M, a.K, a.N, a.es, true);
  l.kp = whole_units(a.K, a.es);
  l.np = packing ? ceil_div(a.N, 8) * 8 : a.N;
  l.need_dz = (a.dx || a.dw) && (a.factor || (packing && (l.np != a.N || !a.g16)));
  if (l.need_dz) l.np = ceil_div(a.N, 8) * 8;
  l.copy_x = packing && a.dw && (l.kp != a.K || !a.x16);
  l.copy_w = packing && a.dx && (l.np != a.N || !a.w16);
  l.w = l.copy_x ? up256((size_t)a.M * l.kp * a.es) : 0;
  l.dz = l.w + (l.copy_w ? up256((size_t)a.K * l.np * a.es) : 0);
  l.sums = l.dz + (l.need_dz ? up256((size_t)a.M * l.np * a.es) : 0);
  l.part = l.sums + (a.db ? up256((size_t)ceil_div(a.M, chunk_rows(a.M, a.N)) * a.N * sizeof(float)) : 0);
  size_t p = 0;
  if (a.dx) p = part_bytes(a.M, a.K, a.N, a.es);
  if (a.dw) p = std::max(p, part_bytes(a.K, a.N, a.M, a.es));
  l.bytes = l.part + p;
  return l;
}

// The products of the calls: x w, dz w^T and x^T dz.  (The copies and dz are 16-byte aligned, as the workspace.)
inline Product forward_product(const LinearSizes& a, const Layout& l) {
  const int64_t lda = l.copy_x ? l.kp : a.K, ldb = l.copy_w ? l.np : a.N;
  return {false, true, a.M, a.N, a.K, lda, ldb, a.M, ldb, l.copy_x || a.x16, l.copy_w || a.w16};
}
inline Product dx_product(const LinearSizes& a, const Layout& l) {
  return {false, false, a.M, a.K, a.N, l.need_dz ? l.np : a.N, l.copy_w ? l.np : a.N, a.M, a.K,
          l.need_dz || a.g16, l.copy_w || a.w16};
}
inline Product dw_product(const LinearSizes& a, const Layout& l) {
  const int64_t lda = l.copy_x ? l.kp : a.K, ldb = l.need_dz ? l.np : a.N;
  return {true, true, a.K, a.N, a.M, lda, ldb, lda, ldb, l.copy_x || a.x16, l.need_dz || a.g16};
}

}  // namespace afno
