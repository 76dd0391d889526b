// afno_mx8.hip -- launches of the operators in eight bits: tensors to mx8.h's format and back, the
// root-mean-square norm, products of rows in eight bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kernels_mx8.h"
#include "kernels_mx8_linear.h"
#include "launch_util.h"
#include "mx8_internal.h"
#include "mx8_rules.h"
#include "train_internal.h"

namespace afno {
namespace {

// a launch's workgroups of 256 threads, which go over `threads` in strides
dim3 strided(int64_t threads) { return dim3((unsigned)std::min<int64_t>(1 << 20, ceil_div(threads, 256))); }

// Workgroups whose waves share the rows of rms_rows_backward: two a CU, of narrow rows four, whose sums for dgamma are
// short (256, 512, 1,024 and 2,048 of them, with the join: 64,800 x 1,024 bf16 136, 99, 115 and 109 us, 16,200 x 2,048 66,
// 67, 74 and 91; 64,800 x 333 86, 51, 42 and 48, 64,800 x 512 100, 62, 53 and 55).
int64_t rms_groups(int64_t M, int64_t C) {
  return std::min<int64_t>(C <= 512 ? 1024 : 512, ceil_div(M * norm_row_waves(C), 4));
}
size_t rms_sums(const RmsBwd& a) {
  const int64_t n = a.C > kNormRowMax ? ceil_div(a.M, chunk_rows(a.M, a.C)) : rms_groups(a.M, a.C);
  return up256((size_t)n * a.C * sizeof(float));
}

}  // namespace

hipError_t launch_pack8(const void* x, const Rows8& o, int64_t M, int64_t C, int dtype, hipStream_t st) {
  return by_type(dtype, [&](auto z) {
    typedef decltype(z) T;
    hipLaunchKernelGGL((mx8_pack_kernel<T>), strided(M * (o.ld / 8)), dim3(256), 0, st,
                       static_cast<const T*>(x), o, M, C);
    return hipGetLastError();
  });
}

hipError_t launch_unpack8(const Rows8& x, void* out, int64_t ldo, int64_t M, int dtype, hipStream_t st) {
  return by_type(dtype, [&](auto z) {
    typedef decltype(z) T;
    by_flag(ldo % 8 == 0 && at16(out), [&](auto v) {
      hipLaunchKernelGGL((mx8_unpack_kernel<T, decltype(v)::value>), strided(M * ceil_div(ldo, 8)), dim3(256), 0,
                         st, x.q, x.s, x.ld, static_cast<T*>(out), ldo, M);
    });
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------- the norm

hipError_t launch_rms_forward(const RmsFwd& a, hipStream_t st) {
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.residual);
    const T* ga = static_cast<const T*>(a.gamma);
    T *out = static_cast<T*>(a.out), *sum = static_cast<T*>(a.sum);
    const bool vec = a.C % Unit<T>::UE == 0 && at16(x) && at16(r) && at16(ga) && at16(out) &&
                     at16(sum);
    if (a.C > kNormRowMax)
      hipLaunchKernelGGL((rms_wide<T>), dim3((unsigned)a.M), dim3(256), 0, st, x, r, ga, out, sum, a.out8, (int)a.C,
                         a.eps);
    else
      by_flag(vec, [&](auto v) {
        by_capacity(a.C, [&](auto cap, auto w) {
          hipLaunchKernelGGL((rms_rows<T, decltype(v)::value, decltype(cap)::value, decltype(w)::value>),
                             dim3((unsigned)ceil_div(a.M, 4 / decltype(w)::value)), dim3(256), 0, st, x, r, ga, out,
                             sum, a.out8, a.M, (int)a.C, a.eps);
        });
      });
    return hipGetLastError();
  });
}

size_t rms_backward_bytes(const RmsBwd& a) {
  return rms_sums(a) + (a.C > kNormRowMax ? (size_t)a.M * sizeof(float) : 0);
}

hipError_t launch_rms_backward(const RmsBwd& a, void* ws, hipStream_t st) {
  if (a.M == 0) {
    fill_zero(a.dgamma, (size_t)a.C * 4, st);
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
      float* stats = reinterpret_cast<float*>(static_cast<char*>(ws) + rms_sums(a));
      const int64_t rows = chunk_rows(a.M, a.C);
      chunks = ceil_div(a.M, rows);
      hipLaunchKernelGGL((rms_wide_backward<T>), dim3((unsigned)a.M), dim3(256), 0, st, g, x, ga, gs, dx, stats,
                         (int)a.C, a.eps);
      hipLaunchKernelGGL((rms_columns<T>), dim3((unsigned)ceil_div(a.C, 256), (unsigned)chunks), dim3(256), 0, st, g,
                         x, stats, part, a.M, (int)a.C, rows);
    } else {
      chunks = rms_groups(a.M, a.C);
      const bool vec = a.C % Unit<T>::UE == 0 && at16(g) && at16(x) && at16(ga) && at16(gs) &&
                       at16(dx);
      by_flag(vec, [&](auto v) {
        by_capacity(a.C, [&](auto cap, auto w) {
          hipLaunchKernelGGL((rms_rows_backward<T, decltype(v)::value, decltype(cap)::value, decltype(w)::value>),
                             dim3((unsigned)chunks), dim3(256), 0, st, g, x, ga, gs, dx, part, a.M, (int)a.C, a.eps);
        });
      });
    }
    hipLaunchKernelGGL((join_columns<float>), dim3((unsigned)ceil_div(a.C, 16)), dim3(1024), 0, st, part, (int)chunks,
                       a.C, a.C, a.dgamma, static_cast<float*>(nullptr));
    return hipGetLastError();
  });
}

// ---------------------------------------------------------------- products

size_t mx8_forward_bytes(const Mx8Fwd& a) { return mx8_part_bytes(a.M, a.N, a.x.ld, a.dtype == 0 ? 4 : 2); }

hipError_t launch_mx8_forward(const Mx8Fwd& a, void* ws, hipStream_t st) {
  return by_type(a.dtype, [&](auto z) {
    typedef decltype(z) T;
    Mx8Args<T> g = {};
    g.a = a.x.q;
    g.as = a.x.s;
    g.b = a.w.q;
    g.bs = a.w.s;
    g.M = a.M;
    g.N = a.N;
    g.ld = a.x.ld;
    g.e = {static_cast<const T*>(a.b), static_cast<const T*>(a.residual), static_cast<T*>(a.out), nullptr, a.act,
           a.drop};
    g.out8 = a.out8;
    g.pre8 = a.pre8;
    if (mx8_few_rows(a.M, a.x.ld)) {
      hipLaunchKernelGGL((mx8_rows<T>), dim3((unsigned)ceil_div(a.N, 32)), dim3(64 * kFewRowsWaves), 0, st, g);
      return hipGetLastError();
    }
    const Cut c = cut_mx8(a.M, a.N, a.x.ld, (int)sizeof(T));
    g.kper = c.kper;
    g.splits = c.splits;
    g.part = c.splits > 1 ? static_cast<float*>(ws) : nullptr;
    const dim3 grid((unsigned)(8 * ceil_div(c.splits * ceil_div(g.M, c.tile) * ceil_div(g.N, c.tile), 8)));
    if constexpr (sizeof(T) == 2) {
      if (c.tile == 256) hipLaunchKernelGGL(mx8_gemm_tile256, grid, dim3(512), 0, st, g);
    }
    if (c.tile == 128) hipLaunchKernelGGL((mx8_gemm_tile<T, 128>), grid, dim3(256), 0, st, g);
    if (c.tile == 64) hipLaunchKernelGGL((mx8_gemm_tile<T, 64>), grid, dim3(256), 0, st, g);
    if (c.splits > 1)
      hipLaunchKernelGGL((mx8_join_splits<T>), dim3((unsigned)ceil_div(g.M * (row8(g.N) / 8), 256)), dim3(256), 0, st,
                         g);
    return hipGetLastError();
  });
}

}  // namespace afno
