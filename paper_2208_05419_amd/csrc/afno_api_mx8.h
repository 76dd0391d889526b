// afno_api_mx8.h -- the C entry points of the operators in eight bits and of the root-mean-square norm: argument
// validation (before any HIP call), workspace and launches.  Part of afno_api.cpp, behind afno_api_train.h.
#pragma once
#include "mx8_internal.h"

namespace {

#define AFNO_TRY(E)                    \
  do {                                 \
    const int rc_ = (E);               \
    if (rc_ != AFNO_OK) return rc_;    \
  } while (0)

// rows of C channels in eight bits at these addresses
afno::Rows8 rows8(const void* values, const void* scales, int64_t C) {
  return {static_cast<uint8_t*>(const_cast<void*>(values)), static_cast<uint8_t*>(const_cast<void*>(scales)),
          afno::row8(C)};
}
Range values_of(const afno::Rows8& r, int64_t M) { return {r.q, (size_t)M * r.ld}; }
Range scales_of(const afno::Rows8& r, int64_t M) { return {r.s, (size_t)M * (r.ld / afno::kBlock8)}; }

// both of its arrays or neither, the values at a 16-byte boundary
int check_rows8(const afno::Rows8& r, bool wanted, const char* name) {
  if (!r.q != !r.s)
    return fail(AFNO_ERR_INVALID_ARG, std::string(name) + ": values and scales come together");
  if (wanted && !r.q) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  if (!aligned(r.q, 16)) return fail(AFNO_ERR_UNSUPPORTED, std::string(name) + ": values must be 16-byte aligned");
  return AFNO_OK;
}

int run_mx8_pack(const void* x, int64_t M, int64_t C, int dtype, void* values, void* scales, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  if (M == 0) return AFNO_OK;
  AFNO_TRY(check_size(M, C));
  const afno::Rows8 o = rows8(values, scales, C);
  if (!x) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_rows8(o, true, "values"));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_aligned({x}, es));
  AFNO_TRY(check_overlap({{x, (size_t)M * C * es}}, {values_of(o, M), scales_of(o, M)}));
  return with_workspace(nullptr, 0, stream, [&](void*) { return afno::launch_pack8(x, o, M, C, dtype, stream); });
}

int run_mx8_unpack(const void* values, const void* scales, int64_t M, int64_t C, int dtype, void* out,
                   hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  if (M == 0) return AFNO_OK;
  AFNO_TRY(check_size(M, C));
  const afno::Rows8 x = rows8(values, scales, C);
  if (!out) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_rows8(x, true, "values"));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_aligned({out}, es));
  AFNO_TRY(check_overlap({values_of(x, M), scales_of(x, M)}, {{out, (size_t)M * C * es}}));
  return with_workspace(nullptr, 0, stream, [&](void*) { return afno::launch_unpack8(x, out, C, M, dtype, stream); });
}

int check_eps(float eps) {
  return eps >= 0.f && std::isfinite(eps) ? AFNO_OK : fail(AFNO_ERR_INVALID_ARG, "eps must be finite and >= 0");
}

int run_rms_forward(const void* x, const void* residual, const void* gamma, int64_t M, int64_t C, float eps, int dtype,
                    void* out, void* sum, void* values, void* scales, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  AFNO_TRY(check_eps(eps));
  if (M == 0) return AFNO_OK;
  AFNO_TRY(check_size(M, C));
  const afno::Rows8 o = rows8(values, scales, C);
  AFNO_TRY(check_rows8(o, !out, "out_values"));
  if (!x || !gamma) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2, n = (size_t)M * C * es;
  AFNO_TRY(check_aligned({x, residual, gamma, out, sum}, es));
  AFNO_TRY(check_overlap({{x, n}, {residual, n}, {gamma, (size_t)C * es}},
                         {{out, n}, {sum, n}, values_of(o, M), scales_of(o, M)}));
  const afno::RmsFwd a{x, residual, gamma, M, C, eps, dtype, out, sum, o};
  return with_workspace(nullptr, 0, stream, [&](void*) { return afno::launch_rms_forward(a, stream); });
}

int run_rms_backward(const void* g, const void* x, const void* gamma, const void* gsum, int64_t M, int64_t C, float eps,
                     int dtype, void* dx, float* dgamma, void* workspace, int64_t workspace_bytes,
                     hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || C <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and C > 0");
  AFNO_TRY(check_eps(eps));
  if (!dgamma || (M > 0 && (!g || !x || !gamma || !dx))) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
  AFNO_TRY(check_size(M, C));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2, n = (size_t)M * C * es, c = (size_t)C * es;
  AFNO_TRY(check_aligned({g, x, gamma, gsum, dx}, es));
  AFNO_TRY(check_aligned({dgamma}, 4));
  AFNO_TRY(check_overlap({{g, n}, {x, n}, {gamma, c}, {gsum, n}}, {{dx, n}, {dgamma, (size_t)C * 4}}));
  const afno::RmsBwd a{g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma};
  const size_t need = M ? afno::rms_backward_bytes(a) : 0;
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {{g, n}, {x, n}, {gamma, c}, {gsum, n}, {dx, n}, {dgamma, (size_t)C * 4}}));
  return with_workspace(workspace, need, stream,
                        [&](void* ws) { return afno::launch_rms_backward(a, ws, stream); });
}

int run_mx8_linear_forward(const void* x_values, const void* x_scales, const void* w_values, const void* w_scales,
                           const void* b, const void* residual, int64_t M, int64_t K, int64_t N, int activation,
                           float p, uint64_t seed, uint64_t offset, const uint64_t* counter, int dtype, void* out,
                           void* out_values, void* out_scales, void* pre_values, void* pre_scales, void* workspace,
                           int64_t workspace_bytes, hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || K <= 0 || N <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and K, N > 0");
  AFNO_TRY(check_activation(activation));
  afno::DropArgs drop = {};
  AFNO_TRY(make_drop(p, seed, offset, counter, &drop));
  if (M == 0) return AFNO_OK;
  AFNO_TRY(check_size(M, N));
  AFNO_TRY(check_size(M, K));
  AFNO_TRY(check_size(N, K));
  const afno::Mx8Fwd a{rows8(x_values, x_scales, K), rows8(w_values, w_scales, K), b, residual, M, K, N, activation,
                       dtype, drop, out, rows8(out_values, out_scales, N), rows8(pre_values, pre_scales, N)};
  AFNO_TRY(check_rows8(a.x, true, "x_values"));
  AFNO_TRY(check_rows8(a.w, true, "w_values"));
  AFNO_TRY(check_rows8(a.out8, !out, "out_values"));
  AFNO_TRY(check_rows8(a.pre8, false, "pre_values"));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2, ob = (size_t)M * N * es;
  AFNO_TRY(check_aligned({b, residual, out}, es));
  const Range xq = values_of(a.x, M), xs = scales_of(a.x, M), wq = values_of(a.w, N), wsc = scales_of(a.w, N);
  const Range oq = values_of(a.out8, M), os = scales_of(a.out8, M), pq = values_of(a.pre8, M),
              ps = scales_of(a.pre8, M);
  AFNO_TRY(check_overlap({xq, xs, wq, wsc, {b, N * es}, {residual, ob}, {counter, 8}}, {{out, ob}, oq, os, pq, ps}));
  const size_t need = afno::mx8_forward_bytes(a);
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {xq, xs, wq, wsc, {b, N * es}, {residual, ob}, {counter, 8}, {out, ob}, oq, os, pq, ps}));
  return with_workspace(workspace, need, stream, [&](void* ws) { return afno::launch_mx8_forward(a, ws, stream); });
}

int run_mx8_linear_backward(const void* g, const void* x_values, const void* x_scales, const void* w,
                            const void* pre_values, const void* pre_scales, int64_t M, int64_t K, int64_t N,
                            int activation, float p, uint64_t seed, uint64_t offset, const uint64_t* counter,
                            int dtype, void* dx, void* dw, void* db, void* workspace, int64_t workspace_bytes,
                            hipStream_t stream) {
  AFNO_TRY(check_dtype(dtype));
  if (M < 0 || K <= 0 || N <= 0) return fail(AFNO_ERR_INVALID_ARG, "M must be >= 0 and K, N > 0");
  AFNO_TRY(check_activation(activation));
  if (activation == AFNO_ACT_NONE) pre_values = pre_scales = nullptr;  // not read
  if (!dw) x_values = x_scales = nullptr;                              // not read
  afno::LinearBwd a{g, nullptr, w, nullptr, M, K, N, activation, dtype, {}, dx, dw, db};
  AFNO_TRY(make_drop(p, seed, offset, counter, &a.drop));
  if (!dx && !dw && !db) return fail(AFNO_ERR_INVALID_ARG, "no gradient is asked for");
  AFNO_TRY(check_size(K, N));
  if (M > 0) {
    if (!g || (dx && !w)) return fail(AFNO_ERR_INVALID_ARG, "null pointer argument");
    AFNO_TRY(check_size(M, N));
    AFNO_TRY(check_size(M, K));
  }
  a.x8 = rows8(x_values, x_scales, K);
  a.pre8 = rows8(pre_values, pre_scales, N);
  AFNO_TRY(check_rows8(a.x8, M > 0 && dw, "x_values"));
  AFNO_TRY(check_rows8(a.pre8, M > 0 && activation != AFNO_ACT_NONE, "pre_values"));
  const size_t es = dtype == AFNO_DTYPE_FP32 ? 4 : 2;
  AFNO_TRY(check_aligned({g, w, dx, dw, db}, es));
  const size_t xb = (size_t)M * K * es, wb = (size_t)K * N * es, ob = (size_t)M * N * es;
  const Range xq = values_of(a.x8, M), xs = scales_of(a.x8, M), pq = values_of(a.pre8, M), ps = scales_of(a.pre8, M);
  AFNO_TRY(check_overlap({{g, ob}, xq, xs, {w, wb}, pq, ps, {counter, 8}}, {{dx, xb}, {dw, wb}, {db, N * es}}));
  if (M == 0 && !dw && !db) return AFNO_OK;
  const size_t need = M ? afno::linear_backward_bytes(a) : 0;
  AFNO_TRY(check_workspace(workspace, workspace_bytes, need,
                           {{g, ob}, xq, xs, {w, wb}, pq, ps, {counter, 8}, {dx, xb}, {dw, wb}, {db, N * es}}));
  return with_workspace(workspace, need, stream,
                        [&](void* ws) { return afno::launch_linear_backward(a, ws, stream); });
}

#undef AFNO_TRY

}  // namespace

extern "C" {

int afno_mx8_pack(const void* x, int64_t M, int64_t C, int dtype, void* values, void* scales, hipStream_t stream) {
  return guarded([&] { return run_mx8_pack(x, M, C, dtype, values, scales, stream); });
}

int afno_mx8_unpack(const void* values, const void* scales, int64_t M, int64_t C, int dtype, void* out,
                    hipStream_t stream) {
  return guarded([&] { return run_mx8_unpack(values, scales, M, C, dtype, out, stream); });
}

int afno_rms_norm_forward(const void* x, const void* residual, const void* gamma, int64_t M, int64_t C, float eps,
                          int dtype, void* out, void* sum, void* out_values, void* out_scales, hipStream_t stream) {
  return guarded([&] {
    return run_rms_forward(x, residual, gamma, M, C, eps, dtype, out, sum, out_values, out_scales, stream);
  });
}

int afno_rms_norm_backward(const void* g, const void* x, const void* gamma, const void* gsum, int64_t M, int64_t C,
                           float eps, int dtype, void* dx, float* dgamma, void* workspace, int64_t workspace_bytes,
                           hipStream_t stream) {
  return guarded([&] {
    return run_rms_backward(g, x, gamma, gsum, M, C, eps, dtype, dx, dgamma, workspace, workspace_bytes, stream);
  });
}

int afno_mx8_linear_forward(const void* x_values, const void* x_scales, const void* w_values, const void* w_scales,
                            const void* b, const void* residual, int64_t M, int64_t K, int64_t N, int activation,
                            float p, uint64_t seed, uint64_t offset, const uint64_t* counter, int dtype, void* out,
                            void* out_values, void* out_scales, void* pre_values, void* pre_scales, void* workspace,
                            int64_t workspace_bytes, hipStream_t stream) {
  return guarded([&] {
    return run_mx8_linear_forward(x_values, x_scales, w_values, w_scales, b, residual, M, K, N, activation, p, seed,
                                  offset, counter, dtype, out, out_values, out_scales, pre_values, pre_scales,
                                  workspace, workspace_bytes, stream);
  });
}

int afno_mx8_linear_backward(const void* g, const void* x_values, const void* x_scales, const void* w,
                             const void* pre_values, const void* pre_scales, int64_t M, int64_t K, int64_t N,
                             int activation, float p, uint64_t seed, uint64_t offset, const uint64_t* counter,
                             int dtype, void* dx, void* dw, void* db, void* workspace, int64_t workspace_bytes,
                             hipStream_t stream) {
  return guarded([&] {
    return run_mx8_linear_backward(g, x_values, x_scales, w, pre_values, pre_scales, M, K, N, activation, p, seed,
                                   offset, counter, dtype, dx, dw, db, workspace, workspace_bytes, stream);
  });
}

int64_t afno_rms_norm_backward_workspace(int64_t M, int64_t C, int dtype) {
  return workspace_of(M, C, 1, dtype, [&] {
    return afno::rms_backward_bytes({nullptr, nullptr, nullptr, nullptr, M, C, 0.f, dtype, nullptr, nullptr});
  });
}

int64_t afno_mx8_linear_forward_workspace(int64_t M, int64_t K, int64_t N, int dtype) {
  return workspace_of(M, K, N, dtype, [&] {
    afno::Mx8Fwd a = {};
    a.x.ld = afno::row8(K);
    a.M = M;
    a.K = K;
    a.N = N;
    a.dtype = dtype;
    return afno::mx8_forward_bytes(a);
  });
}

int64_t afno_mx8_linear_backward_workspace(int64_t M, int64_t K, int64_t N, int dtype, int aligned) {
  return workspace_of(M, K, N, dtype, [&] {
    const void* p = some_address(aligned);
    void* out = const_cast<void*>(p);
    afno::LinearBwd a{p, nullptr, p, nullptr, M, K, N, AFNO_ACT_GELU, dtype, {}, out, out, out};
    a.x8 = rows8(out, out, K);
    a.pre8 = rows8(out, out, N);
    return afno::linear_backward_bytes(a);
  });
}

}  // extern "C"
