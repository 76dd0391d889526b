// mx8_internal.h -- the launchers of afno_mx8.hip that the C ABI and the other launchers call: tensors in eight bits,
// the root-mean-square norm, products of rows in eight bits.  Every pointer has been checked; dtype is 0
// (fp32) or 1 (bf16).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dropout.h"
#include "mx8.h"

namespace afno {

// out = v / sqrt(mean(v^2) + eps) gamma, v = x + residual; residual, out, sum and out8.q may be null.
struct RmsFwd {
  const void *x, *residual, *gamma;
  int64_t M, C;
  float eps;
  int dtype;
  void *out, *sum;
  Rows8 out8;
};
struct RmsBwd {
  const void *g, *x, *gamma, *gsum;
  int64_t M, C;
  float eps;
  int dtype;
  void* dx;
  float* dgamma;
};
// out = drop(act(x w + b)) + residual; b, residual, out, out8.q and pre8.q may be null.
struct Mx8Fwd {
  Rows8 x, w;
  const void *b, *residual;
  int64_t M, K, N;
  int act, dtype;
  DropArgs drop;
  void* out;
  Rows8 out8, pre8;
};

hipError_t launch_pack8(const void* x, const Rows8& o, int64_t M, int64_t C, int dtype, hipStream_t st);
// rows of ldo values, at most the row's ld; zeros behind the channels
hipError_t launch_unpack8(const Rows8& x, void* out, int64_t ldo, int64_t M, int dtype, hipStream_t st);
hipError_t launch_rms_forward(const RmsFwd& a, hipStream_t st);
// workspace bytes (0: none), and the launches with that much at ws
size_t rms_backward_bytes(const RmsBwd& a);
hipError_t launch_rms_backward(const RmsBwd& a, void* ws, hipStream_t st);
size_t mx8_forward_bytes(const Mx8Fwd& a);
hipError_t launch_mx8_forward(const Mx8Fwd& a, void* ws, hipStream_t st);

}  // namespace afno
