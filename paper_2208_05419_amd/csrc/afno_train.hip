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

// How a product is cut: tiles, and splits of k whose sums join_splits adds.
struct Cut {
  int tile;  // 256: gemm_tile256; 128 or 64: gemm_reg's square tile
  int splits;
  int64_t kper;
};

// wide: the operands are what gemm_tile256 takes (bf16, multiples of 8, 16-byte aligned).  It runs one
// workgroup a CU, so it is for products that give most CUs a tile, split over k if need be with 512
// k's at least to each.  Else a tile row or column costs its whole tile, so 128 x 128 where that many
// tiles (times the splits that leave 256 k's to each) give every CU one, else 64 x 64; splits until there
// are two workgroups a CU, each with at least 128 k's.
Cut cut_product(int64_t M, int64_t N, int64_t K, bool wide) {
  Cut c;
  int64_t s;
  if (wide) {
    const int64_t t = ceil_div(M, 256) * ceil_div(N, 256);
    s = t >= 128 ? 1 : std::max<int64_t>(1, std::min<int64_t>(256 / t, K / 512));
    if (t * s >= 128) {
      c.tile = 256;
      c.kper = ceil_div(ceil_div(K, s), 64) * 64;
      c.splits = (int)ceil_div(K, c.kper);
      return c;
    }
  }
  const int64_t t128 = ceil_div(M, 128) * ceil_div(N, 128), t64 = ceil_div(M, 64) * ceil_div(N, 64);
  c.tile = M > 64 && N > 64 && t128 * std::max<int64_t>(1, K / 256) >= 256 ? 128 : 64;
  const int64_t t = c.tile == 128 ? t128 : t64;
  s = std::min<int64_t>(ceil_div(512, t), std::max<int64_t>(1, K / (c.tile == 128 ? 256 : 128)));
  if (t >= 256) s = 1;
  c.kper = std::max<int64_t>(32, ceil_div(ceil_div(K, s), 32) * 32);
  c.splits = (int)std::max<int64_t>(1, ceil_div(K, c.kper));
  return c;
}
size_t part_of(int64_t M, int64_t N, const Cut& c) {
  return c.splits > 1 ? (size_t)c.splits * M * N * sizeof(float) : 0;
}
// whatever the addresses turn out to be
size_t part_bytes(int64_t M, int64_t N, int64_t K, int dtype) {
  const size_t any = part_of(M, N, cut_product(M, N, K, false));
  return dtype == 0 ? any : std::max(any, part_of(M, N, cut_product(M, N, K, true)));
}

template <typename T, bool AR, bool BR, int BM, int BN, bool VEC>
void run_reg(const GemmArgs<T>& g, int splits, hipStream_t st) {
  constexpr int lds = RegGeo<T, AR, BR, BM, BN>::kBytes;
  const int64_t tiles = ceil_div(g.M, BM) * ceil_div(g.N, BN);
  hipLaunchKernelGGL((gemm_reg<T, AR, BR, BM, BN, VEC>),
                     dim3((unsigned)(8 * ceil_div(tiles, 8)), (unsigned)splits), dim3(256),
                     lds, st, g);
}

// One product with its epilogue; part: room for part_bytes.
template <typename T, bool AR, bool BR>
hipError_t product(GemmArgs<T> g, float* part, hipStream_t st) {
  constexpr int UE = Unit<T>::UE;
  const bool vec = g.lda % UE == 0 && g.ldb % UE == 0 && at16(g.a) && at16(g.b);
  // (row-major operands have lda = M and ldb = N, k-major ones K)
  const bool wide = sizeof(T) == 2 && vec && g.N % 8 == 0 && at16(g.e.out) && at16(g.e.pre) &&
                    at16(g.e.residual);
  const Cut c = cut_product(g.M, g.N, g.K, wide);
  g.kper = c.kper;
  g.part = c.splits > 1 ? part : nullptr;
  if (c.tile == 256) {
    if constexpr (sizeof(T) == 2) {
      const int64_t tiles = ceil_div(g.M, 256) * ceil_div(g.N, 256);
      hipLaunchKernelGGL((gemm_tile256<AR, BR>), dim3((unsigned)(8 * ceil_div(tiles, 8)), (unsigned)c.splits),
                         dim3(512), 0, st, g);
    }
  } else by_flag(vec, [&](auto v) {
    constexpr bool V = decltype(v)::value;
    if (c.tile == 128)
      run_reg<T, AR, BR, 128, 128, V>(g, c.splits, st);
    else
      run_reg<T, AR, BR, 64, 64, V>(g, c.splits, st);
  });
  if (c.splits > 1)
    hipLaunchKernelGGL((join_splits<T>), dim3((unsigned)ceil_div(g.M * ceil_div(g.N, 4), 256)),
                       dim3(256), 0, st, part, c.splits, g.M, g.N, g.e);
  return hipGetLastError();
}

// Chunks of rows of the column sums: as many as fill the chip with 256-column workgroups, of at least
// 32 rows.
int64_t chunk_rows(int64_t M, int64_t N) {
  const int64_t want = std::max<int64_t>(1, 1024 / ceil_div(N, 256));
  return std::max<int64_t>(32, ceil_div(ceil_div(M, want), 8) * 8);
}

struct BwdLayout {
  size_t dz, sums, part, bytes;
  bool need_dz;
};
BwdLayout layout(const LinearBwd& a) {
  BwdLayout l = {};
  const size_t es = a.dtype == 0 ? 4 : 2;
  l.need_dz = (a.act != kActNone || a.drop.threshold) && (a.dx || a.dw);
  size_t at = 0;
  l.dz = at;
  if (l.need_dz) at += up256((size_t)a.M * a.N * es);
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

hipError_t set_train_attributes() {
  hipError_t first = hipSuccess;
  auto set = [&](const void* k) {
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess && first == hipSuccess) first = e;
  };
#define AFNO_REG(T, AR, BR)                                                        \
  set(reinterpret_cast<const void*>(&gemm_reg<T, AR, BR, 128, 128, false>));       \
  set(reinterpret_cast<const void*>(&gemm_reg<T, AR, BR, 128, 128, true>));
  AFNO_REG(float, false, true)
  AFNO_REG(float, false, false)
  AFNO_REG(float, true, true)
#undef AFNO_REG
  return first;
}

size_t linear_forward_bytes(const LinearFwd& a) {
  return part_bytes(a.M, a.N, a.K, a.dtype);
}

hipError_t launch_linear_forward(const LinearFwd& a, void* ws, hipStream_t st) {
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    GemmArgs<T> g = {};
    g.a = static_cast<const T*>(a.x);
    g.b = static_cast<const T*>(a.w);
    g.lda = a.K;
    g.ldb = a.N;
    g.M = a.M;
    g.N = a.N;
    g.K = a.K;
    g.e = {static_cast<const T*>(a.b), static_cast<const T*>(a.residual), static_cast<T*>(a.out),
           static_cast<T*>(a.pre), a.act, a.drop};
    return product<T, false, true>(g, static_cast<float*>(ws), st);
  });
}

size_t linear_backward_bytes(const LinearBwd& a) { return layout(a).bytes; }

hipError_t launch_linear_backward(const LinearBwd& a, void* ws, hipStream_t st) {
  if (a.M == 0) {  // sums over no row
    const size_t es = a.dtype == 0 ? 4 : 2;
    if (a.dw) fill_zero(a.dw, (size_t)a.K * a.N * es, st);
    if (a.db) fill_zero(a.db, (size_t)a.N * es, st);
    return hipGetLastError();
  }
  const BwdLayout l = layout(a);
  char* base = static_cast<char*>(ws);
  return by_type(a.dtype, [&](auto z) -> hipError_t {
    typedef decltype(z) T;
    const T *g = static_cast<const T*>(a.g), *pre = static_cast<const T*>(a.pre);
    T* dzw = l.need_dz ? reinterpret_cast<T*>(base + l.dz) : nullptr;
    float* sums = reinterpret_cast<float*>(base + l.sums);
    float* part = reinterpret_cast<float*>(base + l.part);
    const T* dz = l.need_dz ? dzw : g;
    if (l.need_dz || a.db) {
      const int64_t rows = chunk_rows(a.M, a.N), chunks = ceil_div(a.M, rows);
      by_flag(a.N % 8 == 0 && at16(g) && at16(pre), [&](auto v) {
        hipLaunchKernelGGL((dz_kernel<T, decltype(v)::value>),
                           dim3((unsigned)ceil_div(a.N, 256), (unsigned)chunks), dim3(256), 0, st, g,
                           pre, dzw, a.db ? sums : nullptr, a.M, a.N, rows, a.act, a.drop);
      });
      if (a.db)
        hipLaunchKernelGGL((join_columns<T>), dim3((unsigned)ceil_div(a.N, 16)), dim3(256), 0, st, sums,
                           (int)chunks, a.N, a.N, static_cast<T*>(a.db), static_cast<T*>(nullptr));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (a.dx) {
      GemmArgs<T> p = {};
      p.a = dz;
      p.b = static_cast<const T*>(a.w);
      p.lda = p.ldb = a.N;
      p.M = a.M;
      p.N = a.K;
      p.K = a.N;
      p.e.out = static_cast<T*>(a.dx);
      const hipError_t e = product<T, false, false>(p, part, st);
      if (e != hipSuccess) return e;
    }
    if (a.dw) {
      GemmArgs<T> p = {};
      p.a = static_cast<const T*>(a.x);
      p.b = dz;
      p.lda = a.K;
      p.ldb = a.N;
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
        hipLaunchKernelGGL((norm_rows<T, decltype(v)::value>), dim3((unsigned)ceil_div(a.M, 4)),
                           dim3(256), 0, st, x, r, ga, be, out, sum, a.M, (int)a.C, a.eps);
      });
    return hipGetLastError();
  });
}

namespace {
// workgroups whose waves share the rows of norm_rows_backward
int64_t norm_groups(int64_t M) { return std::min<int64_t>(512, ceil_div(M, 4)); }
size_t norm_sums(const NormBwd& a) {
  const int64_t n = a.C > kNormRowMax ? ceil_div(a.M, chunk_rows(a.M, a.C)) : norm_groups(a.M);
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
      chunks = norm_groups(a.M);
      const bool vec = a.C % Unit<T>::UE == 0 && at16(g) && at16(x) && at16(ga) && at16(gs) && at16(dx);
      by_flag(vec, [&](auto v) {
        hipLaunchKernelGGL((norm_rows_backward<T, decltype(v)::value>), dim3((unsigned)chunks), dim3(256),
                           0, st, g, x, ga, gs, dx, part, a.M, (int)a.C, a.eps);
      });
    }
    hipLaunchKernelGGL((join_columns<float>), dim3((unsigned)ceil_div(2 * a.C, 16)), dim3(256), 0, st, part,
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
