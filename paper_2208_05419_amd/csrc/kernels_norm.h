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

constexpr int kNormRowMax = 2048;  // channels a wave holds in registers, 32 a lane

// A lane's part of a row: unit i of UE neighbouring channels from UE (lane + 64 i).  VEC: 16-byte
// units (C a multiple of one, all bases 16-byte aligned); else single channels.
template <typename T, bool VEC>
struct RowPart {
  static constexpr int UE = VEC ? 16 / (int)sizeof(T) : 1, NU = kNormRowMax / 64 / UE;
  __device__ static __forceinline__ void load(const T* p, float (&v)[UE]) {
    if constexpr (VEC) {
      union { uint4 u; T e[UE]; } w;
      w.u = *reinterpret_cast<const uint4*>(p);
#pragma unroll
      for (int e = 0; e < UE; ++e) v[e] = (float)w.e[e];
    } else {
      v[0] = ld_f(p);
    }
  }
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

// mean and 1 / sqrt(var + eps) of a row held by a wave
template <int NU, int UE>
__device__ __forceinline__ void row_stats(const float (&v)[NU][UE], int lane, int units, int C,
                                          float eps, float* mean, float* rstd) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i)
    if (lane + 64 * i < units) {
#pragma unroll
      for (int e = 0; e < UE; ++e) s += v[i][e];
    }
  const float mu = wave_sum(s) / (float)C;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NU; ++i)
    if (lane + 64 * i < units) {
#pragma unroll
      for (int e = 0; e < UE; ++e) {
        const float d = v[i][e] - mu;
        q += d * d;
      }
    }
  *mean = mu;
  *rstd = rsqrtf(wave_sum(q) / (float)C + eps);
}

// C <= kNormRowMax: a wave a row, 4 rows a workgroup.  residual and sum may be null.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_rows(const T* __restrict__ x,
                                                 const T* __restrict__ residual,
                                                 const T* __restrict__ gamma,
                                                 const T* __restrict__ beta, T* __restrict__ out,
                                                 T* __restrict__ sum, int64_t M, int C, float eps) {
  typedef RowPart<T, VEC> P;
  const int lane = threadIdx.x & 63, units = C / P::UE;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= M) return;
  float v[P::NU][P::UE];
#pragma unroll
  for (int i = 0; i < P::NU; ++i) {
    const int c = P::UE * (lane + 64 * i);
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
  row_stats(v, lane, units, C, eps, &mean, &rstd);
#pragma unroll
  for (int i = 0; i < P::NU; ++i) {
    const int c = P::UE * (lane + 64 * i);
    if (c >= C) continue;
    float ga[P::UE], be[P::UE], o[P::UE];
    P::load(gamma + c, ga);
    P::load(beta + c, be);
#pragma unroll
    for (int e = 0; e < P::UE; ++e) o[e] = (v[i][e] - mean) * rstd * ga[e] + be[e];
    P::store(out + m * C + c, o);
  }
}

// C <= kNormRowMax: workgroup b's waves take rows 4 b + wave, then every 4 gridDim.x-th; each lane
// keeps its channels' dgamma and dbeta over its rows, the workgroup adds its waves' in order and
// stores part [gridDim.x][2][C].
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_rows_backward(
    const T* __restrict__ g, const T* __restrict__ x, const T* __restrict__ gamma,
    const T* __restrict__ gsum, T* __restrict__ dx, float* __restrict__ part, int64_t M, int C,
    float eps) {
  typedef RowPart<T, VEC> P;
  __shared__ float sums[2 * kNormRowMax];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, units = C / P::UE;
  float dg[P::NU][P::UE], db[P::NU][P::UE];
#pragma unroll
  for (int i = 0; i < P::NU; ++i)
#pragma unroll
    for (int e = 0; e < P::UE; ++e) dg[i][e] = db[i][e] = 0.f;
  const float inv = 1.f / (float)C;
  for (int64_t m = (int64_t)blockIdx.x * 4 + wave; m < M; m += (int64_t)gridDim.x * 4) {
    float v[P::NU][P::UE], a[P::NU][P::UE];
#pragma unroll
    for (int i = 0; i < P::NU; ++i) {
      const int c = P::UE * (lane + 64 * i);
      if (c >= C) continue;
      P::load(x + m * C + c, v[i]);
      P::load(g + m * C + c, a[i]);
    }
    float mean, rstd, s = 0.f, q = 0.f;
    row_stats(v, lane, units, C, eps, &mean, &rstd);
#pragma unroll
    for (int i = 0; i < P::NU; ++i) {
      const int c = P::UE * (lane + 64 * i);
      if (c >= C) continue;
      float ga[P::UE];
      P::load(gamma + c, ga);
#pragma unroll
      for (int e = 0; e < P::UE; ++e) {
        const float h = (v[i][e] - mean) * rstd;
        v[i][e] = h;
        dg[i][e] += a[i][e] * h;
        db[i][e] += a[i][e];
        a[i][e] *= ga[e];
        s += a[i][e];
        q += a[i][e] * h;
      }
    }
    s = wave_sum(s) * inv;
    q = wave_sum(q) * inv;
#pragma unroll
    for (int i = 0; i < P::NU; ++i) {
      const int c = P::UE * (lane + 64 * i);
      if (c >= C) continue;
      float o[P::UE];
#pragma unroll
      for (int e = 0; e < P::UE; ++e) o[e] = rstd * (a[i][e] - s - v[i][e] * q);
      if (gsum) {
        float r[P::UE];
        P::load(gsum + m * C + c, r);
#pragma unroll
        for (int e = 0; e < P::UE; ++e) o[e] += r[e];
      }
      P::store(dx + m * C + c, o);
    }
  }
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int i = 0; i < P::NU; ++i) {
        const int c = P::UE * (lane + 64 * i);
        if (c >= C) continue;
#pragma unroll
        for (int e = 0; e < P::UE; ++e) {
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

// the sum of v over the workgroup's 256 threads, the same in every thread
__device__ __forceinline__ float group_sum(float v, float* s4) {
  v = wave_sum(v);
  __syncthreads();  // the last sum has been read
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  return s4[0] + s4[1] + s4[2] + s4[3];
}

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
