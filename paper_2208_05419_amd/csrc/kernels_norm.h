// kernels_norm.h -- LayerNorm of a residual sum over the C channels of each of M rows, and its
// gradients:
//   forward   v = x + r, rounded to the storage type;  y = (v - mean) rstd gamma + beta,
//             rstd = 1 / sqrt(var + eps), biased variance
//   backward  with a = g gamma, h = (v - mean) rstd:  dx = rstd (a - mean(a) - h mean(a h)) + gsum,
//             dgamma = sum over the rows of g h,  dbeta = sum over the rows of g
// Statistics in two passes over values held in fp32 (the mean, then the squares about it): the sum of
// squares less the square of the sum loses all digits of a row whose mean is large.  The backward pass
// takes the statistics from v again, which it has to read anyway, so the forward stores none.
#pragma once
#include "kernel_common.h"

namespace afno {

constexpr int kNormRowMax = 8192;  // channels a workgroup holds in registers, 32 a lane

// A lane's part of a row of up to CAP channels that W waves hold: unit i of UE neighbouring channels from
// UE (lane + 64 W i), the lane counted over the W waves.  VEC: 16-byte units (C a multiple of one, all
// bases 16-byte aligned); else single channels.
template <typename T, bool VEC, int CAP, int W>
struct RowPart {
  static constexpr int UE = VEC ? 16 / (int)sizeof(T) : 1, NL = 64 * W, NU = CAP / NL / UE;
  union Raw {
    uint4 u;
    T e[16 / sizeof(T)];
  };
  __device__ static __forceinline__ Raw raw(const T* p) {
    Raw w;
    if constexpr (VEC) w.u = *reinterpret_cast<const uint4*>(p);
    else w.e[0] = *p;
    return w;
  }
  __device__ static __forceinline__ void widen(const Raw& w, float (&v)[UE]) {
#pragma unroll
    for (int e = 0; e < UE; ++e) v[e] = (float)w.e[e];
  }
  __device__ static __forceinline__ void load(const T* p, float (&v)[UE]) { widen(raw(p), v); }
  __device__ static __forceinline__ void store(T* p, const float (&v)[UE]) {
    if constexpr (VEC) {
      union { uint4 u; T e[UE]; } w;
#pragma unroll
      for (int e = 0; e < UE; ++e) w.e[e] = Store<T>::to(v[e]);
      *reinterpret_cast<uint4*>(p) = w.u;
    } else {
      *p = Store<T>::to(v[0]);
    }
  }
};

// the sum of v over the workgroup's 256 threads, the same in every thread
__device__ __forceinline__ float group_sum(float v, float* s4) {
  v = wave_sum(v);
  __syncthreads();  // the last sum has been read
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  return s4[0] + s4[1] + s4[2] + s4[3];
}
// over the W waves of a row
template <int W>
__device__ __forceinline__ float row_sum(float v, float* s4) {
  return W == 1 ? wave_sum(v) : group_sum(v, s4);
}

// mean and 1 / sqrt(var + eps) of a row
template <int W, int NU, int UE>
__device__ __forceinline__ void row_stats(const float (&v)[NU][UE], int lane, int units, int C, float eps,
                                          float* s4, float* mean, float* rstd) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i)
    if (lane + 64 * W * i < units) {
#pragma unroll
      for (int e = 0; e < UE; ++e) s += v[i][e];
    }
  const float mu = row_sum<W>(s, s4) / (float)C;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i)
    if (lane + 64 * W * i < units) {
#pragma unroll
      for (int e = 0; e < UE; ++e) {
        const float d = v[i][e] - mu;
        q += d * d;
      }
    }
  *mean = mu;
  *rstd = rsqrtf(row_sum<W>(q, s4) / (float)C + eps);
}

// C <= CAP: W waves a row, 4 / W rows a workgroup.  residual and sum may be null.
template <typename T, bool VEC, int CAP, int W>
__global__ void __launch_bounds__(256) norm_rows(const T* __restrict__ x,
                                                 const T* __restrict__ residual,
                                                 const T* __restrict__ gamma,
                                                 const T* __restrict__ beta, T* __restrict__ out,
                                                 T* __restrict__ sum, int64_t M, int C, float eps) {
  typedef RowPart<T, VEC, CAP, W> P;
  __shared__ float s4[4];
  const int lane = threadIdx.x & (P::NL - 1), units = C / P::UE;
  const int64_t m = (int64_t)blockIdx.x * (4 / W) + threadIdx.x / P::NL;
  if (m >= M) return;  // whole waves; of W = 4 the whole workgroup
  float v[P::NU][P::UE];
#pragma unroll
  for (int i = 0; i < P::NU; ++i) {
    const int c = P::UE * (lane + P::NL * i);
    if (c >= C) continue;
    P::load(x + m * C + c, v[i]);
    if (residual) {
      float r[P::UE];
      P::load(residual + m * C + c, r);
#pragma unroll
      for (int e = 0; e < P::UE; ++e) v[i][e] = (float)Store<T>::to(v[i][e] + r[e]);
    }
    if (sum) P::store(sum + m * C + c, v[i]);
  }
  float mean, rstd;
  row_stats<W>(v, lane, units, C, eps, s4, &mean, &rstd);
#pragma unroll
  for (int i = 0; i < P::NU; ++i) {
    const int c = P::UE * (lane + P::NL * i);
    if (c >= C) continue;
    float ga[P::UE], be[P::UE], o[P::UE];
    P::load(gamma + c, ga);
    P::load(beta + c, be);
#pragma unroll
    for (int e = 0; e < P::UE; ++e) o[e] = (v[i][e] - mean) * rstd * ga[e] + be[e];
    P::store(out + m * C + c, o);
  }
}

// C <= CAP: workgroup b takes rows 4 / W b and on, then every 4 / W gridDim.x-th, the next row's loads under
// way during the present one's sums (64,800 x 1,024 bf16: 170 us without, 116 with); each lane keeps its
// channels' dgamma and dbeta over its rows, the workgroup adds its rows' in order and stores part
// [gridDim.x][2][C].
template <typename T, bool VEC, int CAP, int W>
__global__ void __launch_bounds__(256) norm_rows_backward(
    const T* __restrict__ g, const T* __restrict__ x, const T* __restrict__ gamma,
    const T* __restrict__ gsum, T* __restrict__ dx, float* __restrict__ part, int64_t M, int C,
    float eps) {
  typedef RowPart<T, VEC, CAP, W> P;
  constexpr int NU = P::NU, UE = P::UE;
  __shared__ float sums[W == 1 ? 2 * CAP : 1];
  __shared__ float s4[4];
  const int lane = threadIdx.x & (P::NL - 1), wave = threadIdx.x / P::NL, units = C / UE;
  float dg[NU][UE], db[NU][UE], ga[NU][UE];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = UE * (lane + P::NL * i);
#pragma unroll
    for (int e = 0; e < UE; ++e) dg[i][e] = db[i][e] = ga[i][e] = 0.f;
    if (c < C) P::load(gamma + c, ga[i]);
  }
  const float inv = 1.f / (float)C;
  const int64_t step = (int64_t)gridDim.x * (4 / W);
  typename P::Raw rv[NU], rg[NU], rs[NU];
  auto fetch = [&](int64_t m) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = UE * (lane + P::NL * i);
      if (c >= C) continue;
      rv[i] = P::raw(x + m * C + c);
      rg[i] = P::raw(g + m * C + c);
      if (gsum) rs[i] = P::raw(gsum + m * C + c);
    }
  };
  int64_t m = (int64_t)blockIdx.x * (4 / W) + wave;
  if (m < M) fetch(m);
  for (; m < M; m += step) {
    float v[NU][UE], a[NU][UE], o[NU][UE];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      P::widen(rv[i], v[i]);
      P::widen(rg[i], a[i]);
#pragma unroll
      for (int e = 0; e < UE; ++e) o[i][e] = 0.f;
      if (gsum) P::widen(rs[i], o[i]);
    }
    if (m + step < M) fetch(m + step);
    float mean, rstd, s = 0.f, q = 0.f;
    row_stats<W>(v, lane, units, C, eps, s4, &mean, &rstd);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      if (lane + P::NL * i >= units) continue;
#pragma unroll
      for (int e = 0; e < UE; ++e) {
        const float h = (v[i][e] - mean) * rstd;
        v[i][e] = h;
        dg[i][e] += a[i][e] * h;
        db[i][e] += a[i][e];
        a[i][e] *= ga[i][e];
        s += a[i][e];
        q += a[i][e] * h;
      }
    }
    s = row_sum<W>(s, s4) * inv;
    q = row_sum<W>(q, s4) * inv;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = UE * (lane + P::NL * i);
      if (c >= C) continue;
#pragma unroll
      for (int e = 0; e < UE; ++e) o[i][e] += rstd * (a[i][e] - s - v[i][e] * q);
      P::store(dx + m * C + c, o[i]);
    }
  }
  if constexpr (W == 4) {
    float* p = part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = UE * (lane + P::NL * i);
      if (c >= C) continue;
#pragma unroll
      for (int e = 0; e < UE; ++e) {
        p[c + e] = dg[i][e];
        p[C + c + e] = db[i][e];
      }
    }
    return;
  }
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int c = UE * (lane + P::NL * i);
        if (c >= C) continue;
#pragma unroll
        for (int e = 0; e < UE; ++e) {
          sums[c + e] = w ? sums[c + e] + dg[i][e] : dg[i][e];
          sums[C + c + e] = w ? sums[C + c + e] + db[i][e] : db[i][e];
        }
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < 2 * C; c += 256) part[(int64_t)blockIdx.x * 2 * C + c] = sums[c];
}

// ---------------------------------------------------------------- wider rows: a workgroup a row

// Rows of any width, read again for each pass (from the caches: 8 KB a row and up).  The backward pass
// leaves (mean, rstd) of each row in stats for norm_columns.
template <typename T>
__global__ void __launch_bounds__(256) norm_wide(const T* __restrict__ x,
                                                 const T* __restrict__ residual,
                                                 const T* __restrict__ gamma,
                                                 const T* __restrict__ beta, T* __restrict__ out,
                                                 T* __restrict__ sum, int C, float eps) {
  __shared__ float s4[4];
  const int64_t base = (int64_t)blockIdx.x * C;
  auto at = [&](int c) {
    const float v = ld_f(x + base + c);
    return residual ? (float)Store<T>::to(v + ld_f(residual + base + c)) : v;
  };
  float s = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float v = at(c);
    if (sum) sum[base + c] = Store<T>::to(v);
    s += v;
  }
  const float mean = group_sum(s, s4) / (float)C;
  float q = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float d = at(c) - mean;
    q += d * d;
  }
  const float rstd = rsqrtf(group_sum(q, s4) / (float)C + eps);
  for (int c = threadIdx.x; c < C; c += 256)
    out[base + c] = Store<T>::to((at(c) - mean) * rstd * ld_f(gamma + c) + ld_f(beta + c));
}

template <typename T>
__global__ void __launch_bounds__(256) norm_wide_backward(const T* __restrict__ g,
                                                          const T* __restrict__ x,
                                                          const T* __restrict__ gamma,
                                                          const T* __restrict__ gsum,
                                                          T* __restrict__ dx,
                                                          float2* __restrict__ stats, int C,
                                                          float eps) {
  __shared__ float s4[4];
  const int64_t base = (int64_t)blockIdx.x * C;
  float s = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) s += ld_f(x + base + c);
  const float mean = group_sum(s, s4) / (float)C;
  float q = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float d = ld_f(x + base + c) - mean;
    q += d * d;
  }
  const float rstd = rsqrtf(group_sum(q, s4) / (float)C + eps);
  if (threadIdx.x == 0) stats[blockIdx.x] = make_float2(mean, rstd);
  float sa = 0.f, sh = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float a = ld_f(g + base + c) * ld_f(gamma + c);
    sa += a;
    sh += a * ((ld_f(x + base + c) - mean) * rstd);
  }
  sa = group_sum(sa, s4) / (float)C;
  sh = group_sum(sh, s4) / (float)C;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float h = (ld_f(x + base + c) - mean) * rstd;
    float o = rstd * (ld_f(g + base + c) * ld_f(gamma + c) - sa - h * sh);
    if (gsum) o += ld_f(gsum + base + c);
    dx[base + c] = Store<T>::to(o);
  }
}

// dgamma and dbeta of a chunk of rows (blockIdx.y), a column a thread: part [chunks][2][C].
template <typename T>
__global__ void __launch_bounds__(256) norm_columns(const T* __restrict__ g, const T* __restrict__ x,
                                                    const float2* __restrict__ stats,
                                                    float* __restrict__ part, int64_t M, int C,
                                                    int64_t rows) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= C) return;
  const int64_t m0 = blockIdx.y * rows, m1 = min(M, m0 + rows);
  float dg = 0.f, db = 0.f;
  for (int64_t m = m0; m < m1; ++m) {
    const float2 st = stats[m];
    const float v = ld_f(g + m * C + c);
    dg += v * ((ld_f(x + m * C + c) - st.x) * st.y);
    db += v;
  }
  part[(int64_t)blockIdx.y * 2 * C + c] = dg;
  part[(int64_t)blockIdx.y * 2 * C + C + c] = db;
}

}  // namespace afno
