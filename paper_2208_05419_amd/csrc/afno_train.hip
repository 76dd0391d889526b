// afno_train.hip -- launches of the operators that train a network around the filter: linear products
// with their epilogue, LayerNorm of a residual sum, dropout.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kernels_linear_dma.h"
#include "kernels_norm.h"
#include "launch_util.h"
#include "linear_rules.h"
#include "mx8_internal.h"
#include "train_internal.h"

namespace afno {
namespace {

__global__ void zero_kernel(uint16_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// ---------------------------------------------------------------- products

// One product with its epilogue, a and b given, the rest of it by p; part: room for part_bytes.
template <typename T, bool AR, bool BR>
hipError_t product(GemmArgs<T> g, const Product& p, float* part, hipStream_t st) {
  g.lda = p.lda;
  g.ldb = p.ldb;
  g.M = p.M;
  g.N = p.N;
  g.K = p.K;
  g.ma = p.ma;
  g.nb = p.nb;
  const Path path = product_path(p, (int)sizeof(T));
  if constexpr (!AR && BR) {
    if (path.rows) {
      const int mr = g.M >= 3 ? 4 : (int)g.M;
      const dim3 grid((unsigned)ceil_div(g.N, kRowsCols), (unsigned)ceil_div(g.M, mr));
      if (mr == 1) hipLaunchKernelGGL((linear_rows<T, 1>), grid, dim3(1024), 0, st, g);
      else if (mr == 2) hipLaunchKernelGGL((linear_rows<T, 2>), grid, dim3(1024), 0, st, g);
      else if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((linear_rows<T, 4>), grid, dim3(1024), 0, st, g);
      return hipGetLastError();
    }
  }
  const Cut& c = path.cut;
  const dim3 grid((unsigned)(8 * ceil_div(c.splits * ceil_div(g.M, c.tile) * ceil_div(g.N, c.tile), 8)));
  g.splits = c.splits;
  g.kper = c.kper;
  g.part = c.splits > 1 ? part : nullptr;
  if (c.tile == 256) {
    if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((gemm_tile256<AR, BR>), grid, dim3(512), 0, st, g);
  } else if (path.units) {
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

template <typename T>
void pack(const PackArgs<T>& a, const PackArgs<T>& b, hipStream_t st) {
  constexpr int UE = Unit<T>::UE;
  const int64_t units = a.rows * (a.ld / UE) + b.rows * (b.ld / UE);
  if (units)
    hipLaunchKernelGGL((pack_rows<T>), dim3((unsigned)std::min<int64_t>(1 << 20, ceil_div(units, 256))), dim3(256),
                       0, st, a, b);
}

LinearSizes sizes_of(const LinearFwd& a) {
  return {a.M, a.K, a.N, a.dtype == 0 ? 4 : 2, at16(a.x), at16(a.w), true, false, false, false, false};
}
LinearSizes sizes_of(const LinearBwd& a) {
  return {a.M, a.K, a.N, a.dtype == 0 ? 4 : 2, at16(a.x), at16(a.w), at16(a.g), a.dx != nullptr, a.dw != nullptr,
          a.db != nullptr, a.act != kActNone || a.drop.threshold != 0, a.x8.q != nullptr};
}

}  // namespace

void fill_zero(void* p, size_t bytes, hipStream_t st) {
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)std::min<size_t>(1024, (bytes / 2 + 255) / 256)), dim3(256),
                     0, st, static_cast<uint16_t*>(p), bytes / 2);
}

size_t linear_forward_bytes(const LinearFwd& a) { return forward_layout(sizes_of(a)).bytes; }

hipError_t launch_linear_forward(const LinearFwd& a, void* ws, hipStream_t st) {
  const LinearSizes sizes = sizes_of(a);
  const Layout l = forward_layout(sizes);
  char* base = static_cast<char*>(ws);
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    GemmArgs<T> g = {};
    g.a = static_cast<const T*>(a.x);
    g.b = static_cast<const T*>(a.w);
    g.e = {static_cast<const T*>(a.b), static_cast<const T*>(a.residual), static_cast<T*>(a.out),
           static_cast<T*>(a.pre), a.act, a.drop};
    PackArgs<T> px = {}, pw = {};
    if (l.copy_x) px = {g.a, reinterpret_cast<T*>(base + l.x), a.M, a.K, l.kp};
    if (l.copy_w) pw = {g.b, reinterpret_cast<T*>(base + l.w), a.K, a.N, l.np};
    pack(px, pw, st);
    if (l.copy_x) g.a = px.dst;
    if (l.copy_w) g.b = pw.dst;
    return product<T, false, true>(g, forward_product(sizes, l),
                                   l.bytes > l.part ? reinterpret_cast<float*>(base + l.part) : nullptr, st);
  });
}

size_t linear_backward_bytes(const LinearBwd& a) { return backward_layout(sizes_of(a)).bytes; }

hipError_t launch_linear_backward(const LinearBwd& a, void* ws, hipStream_t st) {
  if (a.M == 0) {  // sums over no row
    const size_t es = a.dtype == 0 ? 4 : 2;
    if (a.dw) fill_zero(a.dw, (size_t)a.K * a.N * es, st);
    if (a.db) fill_zero(a.db, (size_t)a.N * es, st);
    return hipGetLastError();
  }
  const LinearSizes sizes = sizes_of(a);
  const Layout l = backward_layout(sizes);
  char* base = static_cast<char*>(ws);
  return by_type(a.dtype, [&](auto z) -> hipError_t {
    typedef decltype(z) T;
    const T *g = static_cast<const T*>(a.g), *pre = static_cast<const T*>(a.pre);
    const T *x = static_cast<const T*>(a.x), *w = static_cast<const T*>(a.w);
    T* dzw = l.need_dz ? reinterpret_cast<T*>(base + l.dz) : nullptr;
    float* sums = reinterpret_cast<float*>(base + l.sums);
    float* part = reinterpret_cast<float*>(base + l.part);
    PackArgs<T> px = {}, pw = {};
    if (l.copy_x) px = {x, reinterpret_cast<T*>(base + l.x), a.x8.q ? 0 : a.M, a.K, l.kp};
    if (l.copy_w) pw = {w, reinterpret_cast<T*>(base + l.w), a.K, a.N, l.np};
    pack(px, pw, st);
    // dw's product takes the storage type by transposing reads: 64,800 x 1,024 copied in 36 us of 1,216
    if (a.x8.q && a.dw) {
      const hipError_t e = launch_unpack8(a.x8, px.dst, l.kp, a.M, a.dtype, st);
      if (e != hipSuccess) return e;
    }
    if (l.need_dz || a.db) {
      const int64_t rows = chunk_rows(a.M, a.N), chunks = ceil_div(a.M, rows);
      by_flag(a.N % 8 == 0 && at16(g) && at16(pre), [&](auto v) {
        by_flag(a.pre8.q != nullptr, [&](auto p8) {
          hipLaunchKernelGGL((dz_kernel<T, decltype(v)::value, decltype(p8)::value>),
                             dim3((unsigned)ceil_div(a.N, 256), (unsigned)chunks), dim3(256), 0, st, g, pre, a.pre8,
                             dzw, l.np, a.db ? sums : nullptr, a.M, a.N, rows, a.act, a.drop);
        });
      });
      if (a.db)
        hipLaunchKernelGGL((join_columns<T>), dim3((unsigned)ceil_div(a.N, 16)), dim3(1024), 0, st, sums,
                           (int)chunks, a.N, a.N, static_cast<T*>(a.db), static_cast<T*>(nullptr));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const T* dz = l.need_dz ? dzw : g;
    if (a.dx) {
      GemmArgs<T> p = {};
      p.a = dz;
      p.b = l.copy_w ? pw.dst : w;
      p.e.out = static_cast<T*>(a.dx);
      const hipError_t e = product<T, false, false>(p, dx_product(sizes, l), part, st);
      if (e != hipSuccess) return e;
    }
    if (a.dw) {
      GemmArgs<T> p = {};
      p.a = l.copy_x ? px.dst : x;
      p.b = dz;
      p.e.out = static_cast<T*>(a.dw);
      const hipError_t e = product<T, true, true>(p, dw_product(sizes, l), part, st);
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
        by_capacity(a.C, [&](auto cap, auto w) {
          hipLaunchKernelGGL((norm_rows<T, decltype(v)::value, decltype(cap)::value, decltype(w)::value>),
                             dim3((unsigned)ceil_div(a.M, 4 / decltype(w)::value)), dim3(256), 0, st, x, r, ga, be,
                             out, sum, a.M, (int)a.C, a.eps);
        });
      });
    return hipGetLastError();
  });
}

namespace {
// workgroups whose waves share the rows of norm_rows_backward
int64_t norm_groups(int64_t M, int64_t C) {
  return std::min<int64_t>(C <= 512 ? 1024 : 512, ceil_div(M * norm_row_waves(C), 4));
}
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
