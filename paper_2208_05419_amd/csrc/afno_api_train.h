// afno_api_train.h -- the C entry points of the linear products, LayerNorm and dropout: argument
// validation (before any HIP call), workspace and launches.  Part of afno_api.cpp.
#pragma once
#include <initializer_list>

#include "train_internal.h"

namespace {

struct Range {
  const void* p;
  size_t n;
};

// no output may overlap an input or another output
int check_overlap(std::initializer_list<Range> ins, std::initializer_list<Range> outs) {
  for (const Range& o : outs) {
    if (!o.p || !o.n) continue;
    for (const Range& i : ins)
      if (i.p && i.n && overlaps(o.p, o.n, i.p, i.n))
        return fail(AFNO_ERR_ALIAS, "an output overlaps an input");
    for (const Range& q : outs)
      if (&q != &o && q.p && q.n && overlaps(o.p, o.n, q.p, q.n))
        return fail(AFNO_ERR_ALIAS, "two outputs overlap");
  }
  return AFNO_OK;
}

int check_aligned(std::initializer_list<const void*> ps, size_t es) {
  for (const void* p : ps)
    if (!aligned(p, es)) return fail(AFNO_ERR_UNSUPPORTED, "an array is not aligned to its element size");
  return AFNO_OK;
}

int check_dtype(int dtype) {
  return dtype == AFNO_DTYPE_FP32 || dtype == AFNO_DTYPE_BF16
             ? AFNO_OK
             : fail(AFNO_ERR_INVALID_ARG, "dtype must be AFNO_DTYPE_FP32 (0) or AFNO_DTYPE_BF16 (1)");
}

// The kernels index with 64 bits; a launch has at most 2^32 threads, which these limits keep: a wave a row of
// a norm, 256 threads a tile of 64 x 64, a thread eight values.
constexpr int64_t kMaxWidth = (int64_t)1 << 20, kMaxRows = (int64_t)1 << 25, kMaxValues = (int64_t)1 << 34;
int check_size(int64_t rows, int64_t cols) {
  if (cols > kMaxWidth) return fail(AFNO_ERR_UNSUPPORTED, "more than 2^20 channels");
  if (rows > kMaxRows) return fail(AFNO_ERR_UNSUPPORTED, "more than 2^25 rows");
  if (rows > kMaxValues / cols) return fail(AFNO_ERR_UNSUPPORTED, "more than 2^34 values");
  return AFNO_OK;
}

int make_drop(float p, uint64_t seed, uint64_t offset, const uint64_t* counter, afno::DropArgs* d) {
  if (!(p >= 0.f && p < 1.f)) return fail(AFNO_ERR_INVALID_ARG, "p must be in [0, 1)");
  const double t = std::nearbyint((double)p * 65536.0);
  if (t > 65535.0)
    return fail(AFNO_ERR_INVALID_ARG, "p rounds to 1 in units of 2^-16: nothing would be kept");
  if (!aligned(counter, 8)) return fail(AFNO_ERR_UNSUPPORTED, "counter must be 8-byte aligned");
  *d = afno::DropArgs{seed, offset, counter, (uint32_t)t, (float)(65536.0 / (65536.0 - t))};
  return AFNO_OK;
}

int check_activation(int act) {
  return act == AFNO_ACT_NONE || act == AFNO_ACT_RELU || act == AFNO_ACT_GELU
             ? AFNO_OK
             : fail(AFNO_ERR_INVALID_ARG, "activation must be AFNO_ACT_NONE, AFNO_ACT_RELU or AFNO_ACT_GELU");
}

// the caller's workspace: enough of it, aligned, apart from every array
int check_workspace(const void* ws, int64_t have, size_t need, std::initializer_list<Range> arrays) {
  if (!ws || !need) return AFNO_OK;
  if (have < 0 || (size_t)have < need)
    return fail(AFNO_ERR_INVALID_ARG, "the workspace has " + std::to_string(have) + " bytes of the " +
                                          std::to_string(need) + " that the call needs");
  if (!aligned(ws, 16)) return fail(AFNO_ERR_UNSUPPORTED, "the workspace must be 16-byte aligned");
  for (const Range& r : arrays)
    if (r.p && r.n && overlaps(ws, need, r.p, r.n))
      return fail(AFNO_ERR_ALIAS, "the workspace overlaps an array");
  return AFNO_OK;
}

// The launch with its workspace (bytes == 0: none): the caller's, else one of the library's.  Those
// are not for a captured call: a step has many of these, and a graph takes one call that allocates (acquire()).
template <typename F>
int with_workspace(void* given, size_t bytes, hipStream_t stream, F launch) {
  if (given || !bytes) {
    const hipError_t e = launch(given);
    return e == hipSuccess ? AFNO_OK : fail(AFNO_ERR_HIP, std::string("launch: ") + hipGetErrorString(e));
  }
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(stream, &cap), ef = hipSuccess;
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return fail(AFNO_ERR_HIP, std::string("hipStreamIsCapturing: ") + hipGetErrorString(e));
  }
  if (cap != hipStreamCaptureStatusNone)
    return fail(AFNO_ERR_UNSUPPORTED, "a captured call needs a workspace of the caller's");
  afno::Workspace ws;
  const int rc = acquire(ws, bytes, stream);
  if (rc != AFNO_OK) return rc;
  e = launch(ws.ptr);
  ef = ws.release();
  if (e != hipSuccess) return fail(AFNO_ERR_HIP, std::string("launch: ") + hipGetErrorString(e));
  if (ef != hipSuccess) return fail(AFNO_ERR_HIP, std::string("workspace free: ") + hipGetErrorString(ef));
  return AFNO_OK;
}

#define AFNO_TRY(E)                    \
  do {                                 \
    const int rc_ = (E);               \
    if (rc_ != AFNO_OK) return rc_;    \
  } while (0)

int run_linear_forward(const void* x, const void* w, const void* b, const void* residual, int64_t M,
                       int64_t K, int64_t N, int activation, float p, uint64_t seed, uint64_t offset,
                       const uint64_t* counter, int dtype, void* out, void* pre, void* workspace,
                       int64_t workspace_bytes, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || K <= 0 || N <= 0)
    return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and K, N > 0");
  AFNO_TRY(check_activation(activation));
  afno::LinearFwd a{x, w, b, residual, M, K, N, activation, dtype, {}, out, pre};
  AFNO_TRY(make_drop(p, seed, offset, counter, &a.drop));
  if (M == 0) return AFNO_OK;
  if (!x || !w || !out) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_size(M, N));
  AFNO_TRY(check_size(M, K));
  AFNO_TRY(check_size(K, N));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_aligned({x, w, b, residual, out, pre}, es));
  const size_t xb = (size_t)M * K * es, wb = (size_t)K * N * es, ob = (size_t)M * N * es;
  AFNO_TRY(check_overlap({{x, xb}, {w, wb}, {b, N * es}, {residual, ob}, {counter, 8}},
                         {{out, ob}, {pre, ob}}));
  const size_t need = afno::linear_forward_bytes(a);
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {{x, xb}, {w, wb}, {b, N * es}, {residual, ob}, {counter, 8}, {out, ob}, {pre, ob}}));
  return with_workspace(workspace, need, stream,
                        [&](void* ws) { return afno::launch_linear_forward(a, ws, stream); });
}

int run_linear_backward(const void* g, const void* x, const void* w, const void* pre, int64_t M,
                        int64_t K, int64_t N, int activation, float p, uint64_t seed,
                        uint64_t offset, const uint64_t* counter, int dtype, void* dx, void* dw,
                        void* db, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || K <= 0 || N <= 0)
    return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and K, N > 0");
  AFNO_TRY(check_activation(activation));
  if (activation == AFNO_ACT_NONE) pre = nullptr;  // not read
  afno::LinearBwd a{g, x, w, pre, M, K, N, activation, dtype, {}, dx, dw, db};
  AFNO_TRY(make_drop(p, seed, offset, counter, &a.drop));
  if (!dx && !dw && !db) return fail(AFNO_ERR_INVALID_ARG, "no gradient is asked for");
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_size(K, N));
  if (M > 0) {
    if (!g || (dx && !w) || (dw && !x) || (activation != AFNO_ACT_NONE && !pre))
      return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
    AFNO_TRY(check_size(M, N));
    AFNO_TRY(check_size(M, K));
  }
  AFNO_TRY(check_aligned({g, x, w, pre, dx, dw, db}, es));
  const size_t xb = (size_t)M * K * es, wb = (size_t)K * N * es, ob = (size_t)M * N * es;
  AFNO_TRY(check_overlap({{g, ob}, {x, xb}, {w, wb}, {pre, ob}, {counter, 8}},
                         {{dx, xb}, {dw, wb}, {db, N * es}}));
  if (M == 0 && !dw && !db) return AFNO_OK;
  const size_t need = M ? afno::linear_backward_bytes(a) : 0;
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {{g, ob}, {x, xb}, {w, wb}, {pre, ob}, {counter, 8}, {dx, xb}, {dw, wb}, {db, N * es}}));
  return with_workspace(workspace, need, stream,
                        [&](void* ws) { return afno::launch_linear_backward(a, ws, stream); });
}

int run_norm_forward(const void* x, const void* residual, const void* gamma, const void* beta,
                     int64_t M, int64_t C, float eps, int dtype, void* out, void* sum,
                     hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(AFNO_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (M == 0) return AFNO_OK;
  if (!x || !gamma || !beta || !out) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_size(M, C));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2, n = (size_t)M * C * es, c = (size_t)C * es;
  AFNO_TRY(check_aligned({x, residual, gamma, beta, out, sum}, es));
  AFNO_TRY(check_overlap({{x, n}, {residual, n}, {gamma, c}, {beta, c}}, {{out, n}, {sum, n}}));
  const afno::NormFwd a{x, residual, gamma, beta, M, C, eps, dtype, out, sum};
  return with_workspace(nullptr, 0, stream, [&](void*) { return afno::launch_norm_forward(a, stream); });
}

int run_norm_backward(const void* g, const void* x, const void* gamma, const void* gsum, int64_t M,
                      int64_t C, float eps, int dtype, void* dx, float* dgamma, float* dbeta,
                      void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(AFNO_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!dgamma || !dbeta || (M > 0 && (!g || !x || !gamma || !dx)))
    return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_size(M, C));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2, n = (size_t)M * C * es;
  AFNO_TRY(check_aligned({g, x, gamma, gsum, dx}, es));
  AFNO_TRY(check_aligned({dgamma, dbeta}, 4));
  AFNO_TRY(check_overlap({{g, n}, {x, n}, {gamma, (size_t)C * es}, {gsum, n}},
                         {{dx, n}, {dgamma, (size_t)C * 4}, {dbeta, (size_t)C * 4}}));
  const afno::NormBwd a{g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, dbeta};
  const size_t need = M ? afno::norm_backward_bytes(a) : 0;
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {{g, n}, {x, n}, {gamma, (size_t)C * es}, {gsum, n}, {dx, n},
                            {dgamma, (size_t)C * 4}, {dbeta, (size_t)C * 4}}));
  return with_workspace(workspace, need, stream,
                        [&](void* ws) { return afno::launch_norm_backward(a, ws, stream); });
}

int run_dropout(const void* x, const void* residual, int64_t n, float p, uint64_t seed,
                uint64_t offset, const uint64_t* counter, int dtype, void* out, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (n < 0) return fail(AFNO_ERR_INVALID_ARG, "n must be >= 0");
  afno::DropRunArgs a{x, residual, n, dtype, {}, out};
  AFNO_TRY(make_drop(p, seed, offset, counter, &a.drop));
  if (n == 0) return AFNO_OK;
  if (!x || !out) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  if (n > kMaxValues) return fail(AFNO_ERR_UNSUPPORTED, "more than 2^34 values");
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_aligned({x, residual, out}, es));
  AFNO_TRY(check_overlap({{x, n * es}, {residual, n * es}, {counter, 8}}, {{out, n * es}}));
  return with_workspace(nullptr, 0, stream, [&](void*) { return afno::launch_dropout(a, stream); });
}

#undef AFNO_TRY

// an address for the queries, with every gradient asked for: all that a call of some sizes may need
const void* some_address(int aligned) { return reinterpret_cast<const void*>((uintptr_t)(aligned ? 16 : 4)); }

template <typename F>
int64_t workspace_of(int64_t M, int64_t K, int64_t N, int dtype, F bytes) noexcept try {
  g_last_error.clear();
  int rc = check_dtype(dtype);
  if (rc == AFNO_OK && (M < 0 || K <= 0 || N <= 0)) rc = fail(AFNO_ERR_INVALID_ARG, "sizes must be positive");
  if (rc == AFNO_OK) rc = check_size(M, N);
  if (rc == AFNO_OK) rc = check_size(M, K);
  if (rc == AFNO_OK) rc = check_size(K, N);
  if (rc != AFNO_OK) return rc;
  return M ? (int64_t)bytes() : 0;
} catch (...) {
  return AFNO_ERR_HIP;
}

// no C++ exception (of an allocation for an error's text, of a mutex) passes a C entry
template <typename F>
int guarded(F f) noexcept {
  try {
    g_last_error.clear();
    return f();
  } catch (...) {
    return AFNO_ERR_HIP;
  }
}

}  // namespace

extern "C" {

int afno_linear_forward(const void* x, const void* w, const void* b, const void* residual, int64_t M,
                        int64_t K, int64_t N, int activation, float p, uint64_t seed,
                        uint64_t offset, const uint64_t* counter, int dtype, void* out, void* pre,
                        void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    return run_linear_forward(x, w, b, residual, M, K, N, activation, p, seed, offset, counter, dtype,
                              out, pre, workspace, workspace_bytes, stream);
  });
}

int afno_linear_backward(const void* g, const void* x, const void* w, const void* pre, int64_t M,
                         int64_t K, int64_t N, int activation, float p, uint64_t seed,
                         uint64_t offset, const uint64_t* counter, int dtype, void* dx, void* dw,
                         void* db, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    return run_linear_backward(g, x, w, pre, M, K, N, activation, p, seed, offset, counter, dtype, dx,
                               dw, db, workspace, workspace_bytes, stream);
  });
}

int afno_layer_norm_forward(const void* x, const void* residual, const void* gamma, const void* beta,
                            int64_t M, int64_t C, float eps, int dtype, void* out, void* sum,
                            hipStream_t stream) {
  return guarded([&] {
    return run_norm_forward(x, residual, gamma, beta, M, C, eps, dtype, out, sum, stream);
  });
}

int afno_layer_norm_backward(const void* g, const void* x, const void* gamma, const void* gsum,
                             int64_t M, int64_t C, float eps, int dtype, void* dx, float* dgamma,
                             float* dbeta, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream) {
  return guarded([&] {
    return run_norm_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, dbeta, workspace,
                             workspace_bytes, stream);
  });
}

int afno_dropout_forward(const void* x, const void* residual, int64_t n, float p, uint64_t seed,
                         uint64_t offset, const uint64_t* counter, int dtype, void* out,
                         hipStream_t stream) {
  return guarded([&] {
    return run_dropout(x, residual, n, p, seed, offset, counter, dtype, out, stream);
  });
}

int afno_dropout_backward(const void* g, int64_t n, float p, uint64_t seed, uint64_t offset,
                          const uint64_t* counter, int dtype, void* dx, hipStream_t stream) {
  return guarded([&] {
    return run_dropout(g, nullptr, n, p, seed, offset, counter, dtype, dx, stream);
  });
}

int64_t afno_linear_forward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned) {
  return workspace_of(M, K, N, dtype, [&] {
    const void* p = some_address(aligned);
    return afno::linear_forward_bytes({p, p, nullptr, nullptr, M, K, N, 0, dtype, {}, nullptr, nullptr});
  });
}

int64_t afno_linear_backward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned) {
  return workspace_of(M, K, N, dtype, [&] {
    const void* p = some_address(aligned);
    void* out = const_cast<void*>(p);
    return afno::linear_backward_bytes({p, p, p, p, M, K, N, AFNO_ACT_GELU, dtype, {}, out, out, out});
  });
}

int64_t afno_layer_norm_backward_workspace(int64_t M, int64_t C, int dtype) {
  return workspace_of(M, C, 1, dtype, [&] {
    return afno::norm_backward_bytes({nullptr, nullptr, nullptr, nullptr, M, C, 0.f, dtype, nullptr, nullptr, nullptr});
  });
}

}  // extern "C"
