// afno_train.hip -- launches of the operators that train a network around the filter: linear products
// with their epilogue, LayerNorm of a residual sum, dropout.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "kernels_linear_dma.h"
#include "kernels_norm.h"
#include "train_internal.h"

namespace afno {
namespace {

template <typename F>
auto by_type(int dtype, F f) {
  return dtype == 0 ? f(float()) : f(bf16());
}
template <typename F>
auto by_flag(bool v, F f) {
  return v ? f(std::true_type()) : f(std::false_type());
}
bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }  // null counts as aligned
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// bytes (a multiple of 2, as the address) set to 0: a kernel, so that it replays in a graph
__global__ void zero_kernel(uint16_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}
void fill_zero(void* p, size_t bytes, hipStream_t st) {
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::min<size_t>(1024, (bytes / 2 + 255) / 256)), dim3(256),
                     0, st, static_cast<uint16_t*>(p), bytes / 2);
}

// ---------------------------------------------------------------- products

// How a product is cut: the kernel's square tile, and splits of k whose sums join_splits adds.
struct Cut {
  int tile;  // 256: gemm_tile256; 128 or 64: gemm_tile, or gemm_reg where the operands are no 16-byte units
  int splits;
  int64_t kper;
};

// units: the operands are what the direct-to-LDS kernels take.
// bf16: 256 where most CUs get a tile of it, also by a split of k that leaves 2,048 to each (64,800 k's, 1,024
// x 4,096: 520 us in four splits of 256 against 693 in two of 128; 1,080 x 1,536 x 768, 30 tiles: 20 against
// 8 with 64).  Both: 128 where every CU gets one (bf16, 4,096 x 1,024 x 1,024, 256 tiles: 16.5 us, 64
// 16.6; 10,368 x 1,536 x 384, 972 tiles: 22 and 32; fp32 from three in four: 10,368 x 384 x 1,536, 243
// tiles: 116 and 122), or by splits of long sums (bf16, 10,368 k's in 384 x 1,536: 35 us in eight of 128, 41
// with 64 whole), in fp32 two to a CU where 2,048 k's are left to each (20,000 k's, 2,048 x 2,048: 1,291 us
// in two splits, 1,549 whole; but 10,368 k's in 384 x 1,536: 123 in seven, 152 in ten).
// Else 64, split where the tiles leave CUs without one and the sum is long: a split costs the join's launch,
// about 3 us, and a stage of k's 0.2 us, in fp32 0.7 (bf16, 256 x 1,024 x 4,096, 64 tiles: 16.6 us whole,
// 13.0 in four; 64 x 4,096 x 1,024: 6.3 whole, 8.7 in two; fp32 23.7 whole, 12.9 in four).
// Without units every k-stage waits for its loads: splits until there are two workgroups a CU.
Cut cut_product(int64_t M, int64_t N, int64_t K, int es, bool units) {
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
size_t part_of(int64_t M, int64_t N, const Cut& c) {
  return c.splits > 1 ? (size_t)c.splits * M * N * sizeof(float) : 0;
}
// Whether linear_rows takes a forward product.  bf16, 1,024 x 4,096: 3.9 us for one row, 4.5 for two, 6.0 for
// four, where gemm_tile takes 6.5 for any; fp32 5.2 for eight, 9 for sixteen against 12.
bool few_rows(int64_t M, int es) { return M <= (es == 2 ? 2 : 16); }
// whatever the addresses turn out to be
size_t part_bytes(int64_t M, int64_t N, int64_t K, int dtype) {
  const int es = dtype == 0 ? 4 : 2;
  return std::max(part_of(M, N, cut_product(M, N, K, es, false)), part_of(M, N, cut_product(M, N, K, es, true)));
}

// One product with its epilogue; part: room for part_bytes.  Operands at any address and stride: the
// direct-to-LDS kernels where both are 16-byte units, else gemm_reg.
template <typename T, bool AR, bool BR>
hipError_t product(GemmArgs<T> g, float* part, hipStream_t st) {
  constexpr int UE = Unit<T>::UE;
  if constexpr (!AR && BR) {
    if (few_rows(g.M, (int)sizeof(T))) {
      const int mr = g.M >= 3 ? 4 : (int)g.M;
      const dim3 grid((unsigned)ceil_div(g.N, kRowsCols), (unsigned)ceil_div(g.M, mr));
      if (mr == 1) hipLaunchKernelGGL((linear_rows<T, 1>), grid, dim3(1024), 0, st, g);
      else if (mr == 2) hipLaunchKernelGGL((linear_rows<T, 2>), grid, dim3(1024), 0, st, g);
      else if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((linear_rows<T, 4>), grid, dim3(1024), 0, st, g);
      return hipGetLastError();
    }
  }
  const bool units = g.lda % UE == 0 && g.ldb % UE == 0 && at16(g.a) && at16(g.b) &&
                     (!AR || g.ma % UE == 0) && (!BR || g.nb % UE == 0);
  const Cut c = cut_product(g.M, g.N, g.K, (int)sizeof(T), units);
  const dim3 grid((unsigned)(8 * ceil_div(c.splits * ceil_div(g.M, c.tile) * ceil_div(g.N, c.tile), 8)));
  g.splits = c.splits;
  g.kper = c.kper;
  g.part = c.splits > 1 ? part : nullptr;
  if (c.tile == 256) {
    if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((gemm_tile256<AR, BR>), grid, dim3(512), 0, st, g);
  } else if (units) {
    if (c.tile == 128) hipLaunchKernelGGL((gemm_tile<T, AR, BR, 128>), grid, dim3(TileWaves<T>::NT), 0, st, g);
    else hipLaunchKernelGGL((gemm_tile<T, AR, BR, 64>), grid, dim3(TileWaves<T>::NT), 0, st, g);
  } else {
    if (c.tile == 128) hipLaunchKernelGGL((gemm_reg<T, AR, BR, 128, 128>), grid, dim3(256), 0, st, g);
    else hipLaunchKernelGGL((gemm_reg<T, AR, BR, 64, 64>), grid, dim3(256), 0, st, g);
  }
  if (c.splits > 1)
    hipLaunchKernelGGL((join_splits<T>), dim3((unsigned)ceil_div(g.M * ceil_div(g.N, 4), 256)),
                       dim3(256), 0, st, part, c.splits, g.M, g.N, g.e);
  return hipGetLastError();
}

// Whether operands that are no 16-byte units are copied to rows that are, for the direct-to-LDS kernels: a
// launch and a pass over them, against loads through registers.  bf16: 2,001 x 1,001 x 999 20 us, not
// copied 46; 300 x 77 x 333 7.6 and 6.3, but its gradients, whose factor dz comes in such rows anyway, 20 and 26.
// fp32, whose matrix instructions take longer than the loads: 54 and 74, but 1,000 x 1,001 x 501 27 and
// 27, and 64,800 x 77 x 1,023 with few operations to a byte 242 and 215.
bool worth_packing(int64_t M, int64_t K, int64_t N, int es, bool backward) {
  const double work = (double)M * (double)K * (double)N;
  if (es == 2) return work >= (backward ? 1 << 22 : 1 << 26);
  return work >= 1 << 30 && std::min(K, N) >= 256;
}
template <typename T>
void pack(const PackArgs<T>& a, const PackArgs<T>& b, hipStream_t st) {
  constexpr int UE = Unit<T>::UE;
  const int64_t units = a.rows * (a.ld / UE) + b.rows * (b.ld / UE);
  if (units)
    hipLaunchKernelGGL((pack_rows<T>), dim3((unsigned)std::min<int64_t>(1 << 20, ceil_div(units, 256))), dim3(256),
                       0, st, a, b);
}
int64_t whole_units(int64_t n, int es) { return ceil_div(n, 16 / es) * (16 / es); }

// Chunks of rows of the column sums: as many as fill the chip eight times with 256-column workgroups, of at
// least eight rows, one to a thread (1,080 x 1,536: 11.3 us with 32, 8.1 with eight).
int64_t chunk_rows(int64_t M, int64_t N) {
  const int64_t want = std::max<int64_t>(1, 2048 / ceil_div(N, 256));
  return std::max<int64_t>(8, ceil_div(ceil_div(M, want), 8) * 8);
}

// A call's workspace: copies of operands that are no 16-byte units (whatever the addresses turn out to be,
// room for them where the sizes are worth it), the factor dz, chunk sums, the splits' sums.
struct Layout {
  bool packing, need_dz;
  int64_t kp, np;  // rows of the copies and of dz
  size_t x, w, dz, sums, part, bytes;
};
Layout forward_layout(const LinearFwd& a) {
  Layout l = {};
  const int es = a.dtype == 0 ? 4 : 2;
  if (few_rows(a.M, es)) return l;
  l.packing = worth_packing(a.M, a.K, a.N, es, false);
  l.kp = whole_units(a.K, es);
  l.np = whole_units(a.N, es);
  size_t at = 0;
  l.x = at;
  if (l.packing && (l.kp != a.K || !at16(a.x))) at += up256((size_t)a.M * l.kp * es);
  l.w = at;
  if (l.packing && (l.np != a.N || !at16(a.w))) at += up256((size_t)a.K * l.np * es);
  l.part = at;
  l.bytes = at + part_bytes(a.M, a.N, a.K, a.dtype);
  return l;
}
Layout backward_layout(const LinearBwd& a) {
  Layout l = {};
  const int es = a.dtype == 0 ? 4 : 2;
  l.packing = worth_packing(a.M, a.K, a.N, es, true);
  l.kp = whole_units(a.K, es);
  l.np = l.packing ? ceil_div(a.N, 8) * 8 : a.N;
  l.need_dz = (a.dx || a.dw) &&
              (a.act != kActNone || a.drop.threshold || (l.packing && (l.np != a.N || !at16(a.g))));
  if (l.need_dz) l.np = ceil_div(a.N, 8) * 8;
  size_t at = 0;
  l.x = at;
  if (l.packing && a.dw && (l.kp != a.K || !at16(a.x))) at += up256((size_t)a.M * l.kp * es);
  l.w = at;
  if (l.packing && a.dx && (l.np != a.N || !at16(a.w))) at += up256((size_t)a.K * l.np * es);
  l.dz = at;
  if (l.need_dz) at += up256((size_t)a.M * l.np * es);
  l.sums = at;
  if (a.db) at += up256((size_t)ceil_div(a.M, chunk_rows(a.M, a.N)) * a.N * sizeof(float));
  l.part = at;
  size_t p = 0;
  if (a.dx) p = part_bytes(a.M, a.K, a.N, a.dtype);
  if (a.dw) p = std::max(p, part_bytes(a.K, a.N, a.M, a.dtype));
  l.bytes = at + p;
  return l;
}

}  // namespace

size_t linear_forward_bytes(const LinearFwd& a) { return forward_layout(a).bytes; }

hipError_t launch_linear_forward(const LinearFwd& a, void* ws, hipStream_t st) {
  const Layout l = forward_layout(a);
  char* base = static_cast<char*>(ws);
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    GemmArgs<T> g = {};
    g.a = static_cast<const T*>(a.x);
    g.b = static_cast<const T*>(a.w);
    g.lda = a.K;
    g.ldb = a.N;
    g.M = g.ma = a.M;
    g.N = g.nb = a.N;
    g.K = a.K;
    g.e = {static_cast<const T*>(a.b), static_cast<const T*>(a.residual), static_cast<T*>(a.out),
           static_cast<T*>(a.pre), a.act, a.drop};
    PackArgs<T> px = {}, pw = {};
    if (l.w != l.x) px = {g.a, reinterpret_cast<T*>(base + l.x), a.M, a.K, l.kp};
    if (l.part != l.w) pw = {g.b, reinterpret_cast<T*>(base + l.w), a.K, a.N, l.np};
    pack(px, pw, st);
    if (px.rows) {
      g.a = px.dst;
      g.lda = l.kp;
    }
    if (pw.rows) {
      g.b = pw.dst;
      g.ldb = g.nb = l.np;
    }
    return product<T, false, true>(g, l.bytes > l.part ? reinterpret_cast<float*>(base + l.part) : nullptr, st);
  });
}

size_t linear_backward_bytes(const LinearBwd& a) { return backward_layout(a).bytes; }

hipError_t launch_linear_backward(const LinearBwd& a, void* ws, hipStream_t st) {
  if (a.M == 0) {  // sums over no row
    const size_t es = a.dtype == 0 ? 4 : 2;
    if (a.dw) fill_zero(a.dw, (size_t)a.K * a.N * es, st);
    if (a.db) fill_zero(a.db, (size_t)a.N * es, st);
    return hipGetLastError();
  }
  const Layout l = backward_layout(a);
  char* base = static_cast<char*>(ws);
  return by_type(a.dtype, [&](auto z) -> hipError_t {
    typedef decltype(z) T;
    const T *g = static_cast<const T*>(a.g), *pre = static_cast<const T*>(a.pre);
    const T *x = static_cast<const T*>(a.x), *w = static_cast<const T*>(a.w);
    T* dzw = l.need_dz ? reinterpret_cast<T*>(base + l.dz) : nullptr;
    float* sums = reinterpret_cast<float*>(base + l.sums);
    float* part = reinterpret_cast<float*>(base + l.part);
    PackArgs<T> px = {}, pw = {};
    if (l.w != l.x) px = {x, reinterpret_cast<T*>(base + l.x), a.M, a.K, l.kp};
    if (l.dz != l.w) pw = {w, reinterpret_cast<T*>(base + l.w), a.K, a.N, l.np};
    pack(px, pw, st);
    if (l.need_dz || a.db) {
      const int64_t rows = chunk_rows(a.M, a.N), chunks = ceil_div(a.M, rows);
      by_flag(a.N % 8 == 0 && at16(g) && at16(pre), [&](auto v) {
        hipLaunchKernelGGL((dz_kernel<T, decltype(v)::value>),
                           dim3((unsigned)ceil_div(a.N, 256), (unsigned)chunks), dim3(256), 0, st, g, pre,
                           dzw, l.np, a.db ? sums : nullptr, a.M, a.N, rows, a.act, a.drop);
      });
      if (a.db)
        hipLaunchKernelGGL((join_columns<T>), dim3((unsigned)ceil_div(a.N, 16)), dim3(1024), 0, st, sums,
                           (int)chunks, a.N, a.N, static_cast<T*>(a.db), static_cast<T*>(nullptr));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const T* dz = l.need_dz ? dzw : g;
    const int64_t ldz = l.need_dz ? l.np : a.N;
    if (a.dx) {
      GemmArgs<T> p = {};
      p.a = dz;
      p.lda = ldz;
      p.b = pw.rows ? pw.dst : w;
      p.ldb = pw.rows ? l.np : a.N;
      p.M = p.ma = a.M;
      p.N = p.nb = a.K;
      p.K = a.N;
      p.e.out = static_cast<T*>(a.dx);
      const hipError_t e = product<T, false, false>(p, part, st);
      if (e != hipSuccess) return e;
    }
    if (a.dw) {
      GemmArgs<T> p = {};
      p.a = px.rows ? px.dst : x;
      p.lda = p.ma = px.rows ? l.kp : a.K;
      p.b = dz;
      p.ldb = p.nb = ldz;
      p.M = a.K;
      p.N = a.N;
      p.K = a.M;
      p.e.out = static_cast<T*>(a.dw);
      const hipError_t e = product<T, true, true>(p, part, st);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

// ---------------------------------------------------------------- LayerNorm

namespace {
// the kernels that hold a row in registers, by the channels that they have room for and the waves that
// share a row: all of a row's loads are under way at once, and fewer registers leave more rows to a CU
template <typename F>
void by_capacity(int64_t C, F f) {
  const auto one = std::integral_constant<int, 1>();
  const auto four = std::integral_constant<int, 4>();
  if (C <= 512) f(std::integral_constant<int, 512>(), one);
  else if (C <= 1024) f(std::integral_constant<int, 1024>(), one);
  else if (C <= 2048) f(std::integral_constant<int, 2048>(), one);
  else if (C <= 4096) f(std::integral_constant<int, 4096>(), four);
  else f(std::integral_constant<int, kNormRowMax>(), four);
}
int64_t norm_row_waves(int64_t C) { return C <= 2048 ? 1 : 4; }
}  // namespace

hipError_t launch_norm_forward(const NormFwd& a, hipStream_t st) {
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.residual);
    const T *ga = static_cast<const T*>(a.gamma), *be = static_cast<const T*>(a.beta);
    T *out = static_cast<T*>(a.out), *sum = static_cast<T*>(a.sum);
    const bool vec = a.C % Unit<T>::UE == 0 && at16(x) && at16(r) && at16(ga) && at16(be) &&
                     at16(out) && at16(sum);
    if (a.C > kNormRowMax)
      hipLaunchKernelGGL((norm_wide<T>), dim3((unsigned)a.M), dim3(256), 0, st, x, r, ga, be, out, sum,
                         (int)a.C, a.eps);
    else
      by_flag(vec, [&](auto v) {
        by_capacity(a.C, [&](auto cap, auto w) {
          hipLaunchKernelGGL((norm_rows<T, decltype(v)::value, decltype(cap)::value, decltype(w)::value>),
                             dim3((unsigned)ceil_div(a.M, 4 / decltype(w)::value)), dim3(256), 0, st, x, r, ga, be, out, sum, a.M,
                             (int)a.C, a.eps);
        });
      });
    return hipGetLastError();
  });
}

namespace {
// workgroups whose waves share the rows of norm_rows_backward
int64_t norm_groups(int64_t M, int64_t C) { return std::min<int64_t>(C <= 512 ? 1024 : 512, ceil_div(M * norm_row_waves(C), 4)); }
size_t norm_sums(const NormBwd& a) {
  const int64_t n = a.C > kNormRowMax ? ceil_div(a.M, chunk_rows(a.M, a.C)) : norm_groups(a.M, a.C);
  return up256((size_t)n * 2 * a.C * sizeof(float));
}
}  // namespace

size_t norm_backward_bytes(const NormBwd& a) {
  return norm_sums(a) + (a.C > kNormRowMax ? (size_t)a.M * sizeof(float2) : 0);
}

hipError_t launch_norm_backward(const NormBwd& a, void* ws, hipStream_t st) {
  if (a.M == 0) {
    fill_zero(a.dgamma, (size_t)a.C * 4, st);
    fill_zero(a.dbeta, (size_t)a.C * 4, st);
    return hipGetLastError();
  }
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    const T *g = static_cast<const T*>(a.g), *x = static_cast<const T*>(a.x);
    const T *ga = static_cast<const T*>(a.gamma), *gs = static_cast<const T*>(a.gsum);
    T* dx = static_cast<T*>(a.dx);
    float* part = static_cast<float*>(ws);
    int64_t chunks;
    if (a.C > kNormRowMax) {
      float2* stats = reinterpret_cast<float2*>(static_cast<char*>(ws) + norm_sums(a));
      const int64_t rows = chunk_rows(a.M, a.C);
      chunks = ceil_div(a.M, rows);
      hipLaunchKernelGGL((norm_wide_backward<T>), dim3((unsigned)a.M), dim3(256), 0, st, g, x, ga, gs, dx,
                         stats, (int)a.C, a.eps);
      hipLaunchKernelGGL((norm_columns<T>), dim3((unsigned)ceil_div(a.C, 256), (unsigned)chunks),
                         dim3(256), 0, st, g, x, stats, part, a.M, (int)a.C, rows);
    } else {
      chunks = norm_groups(a.M, a.C);
      const bool vec = a.C % Unit<T>::UE == 0 && at16(g) && at16(x) && at16(ga) && at16(gs) && at16(dx);
      by_flag(vec, [&](auto v) {
        by_capacity(a.C, [&](auto cap, auto w) {
          hipLaunchKernelGGL((norm_rows_backward<T, decltype(v)::value, decltype(cap)::value, decltype(w)::value>),
                             dim3((unsigned)chunks), dim3(256), 0, st, g, x, ga, gs, dx, part, a.M, (int)a.C,
                             a.eps);
        });
      });
    }
    hipLaunchKernelGGL((join_columns<float>), dim3((unsigned)ceil_div(2 * a.C, 16)), dim3(1024), 0, st, part,
                       (int)chunks, 2 * a.C, a.C, a.dgamma, a.dbeta);
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------- dropout

hipError_t launch_dropout(const DropRunArgs& a, hipStream_t st) {
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.residual);
    T* out = static_cast<T*>(a.out);
    by_flag(at16(x) && at16(r) && at16(out), [&](auto v) {
      hipLaunchKernelGGL((dropout_kernel<T, decltype(v)::value>), dim3((unsigned)ceil_div(a.n, 2048)),
                         dim3(256), 0, st, x, r, out, a.n, a.drop);
    });
    return hipGetLastError();
  });
}

}  // namespace afno
