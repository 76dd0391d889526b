// train_internal.h -- the launchers of afno_train.hip that the C ABI calls: linear products, LayerNorm
// and dropout.  Every pointer has been checked; dtype is 0 (fp32) or 1 (bf16).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dropout.h"

namespace afno {

// out = drop(act(x w + b)) + residual; b, residual and pre may be null.
struct LinearFwd {
  const void *x, *w, *b, *residual;
  int64_t M, K, N;
  int act, dtype;
  DropArgs drop;
  void *out, *pre;
};
// Gradients of drop(act(x w + b)) for g; dx, dw and db may be null.
struct LinearBwd {
  const void *g, *x, *w, *pre;
  int64_t M, K, N;
  int act, dtype;
  DropArgs drop;
  void *dx, *dw, *db;
};
struct NormFwd {
  const void *x, *residual, *gamma, *beta;
  int64_t M, C;
  float eps;
  int dtype;
  void *out, *sum;
};
struct NormBwd {
  const void *g, *x, *gamma, *gsum;
  int64_t M, C;
  float eps;
  int dtype;
  void* dx;
  float *dgamma, *dbeta;
};
struct DropRunArgs {
  const void *x, *residual;
  int64_t n;
  int dtype;
  DropArgs drop;
  void* out;
};

// bytes > 0 (a multiple of 2, as the address) set to 0: a kernel, since a graph's memset nodes have not
// replayed reliably
void fill_zero(void* p, size_t bytes, hipStream_t st);
// workspace bytes (0: none), and the launches with that much at ws
size_t linear_forward_bytes(const LinearFwd& a);
hipError_t launch_linear_forward(const LinearFwd& a, void* ws, hipStream_t st);
size_t linear_backward_bytes(const LinearBwd& a);
hipError_t launch_linear_backward(const LinearBwd& a, void* ws, hipStream_t st);
hipError_t launch_norm_forward(const NormFwd& a, hipStream_t st);
size_t norm_backward_bytes(const NormBwd& a);
hipError_t launch_norm_backward(const NormBwd& a, void* ws, hipStream_t st);
hipError_t launch_dropout(const DropRunArgs& a, hipStream_t st);

}  // namespace afno
