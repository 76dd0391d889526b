// kernels_mx8.h -- tensors to eight bits and back, and the root-mean-square norm of a residual sum, whose
// result may be in eight bits (mx8.h), with its gradients:
//   forward   v = x + r, rounded to the storage type;  y = v rms gamma,  rms = 1 / sqrt(mean(v^2) + eps)
//   backward  with a = g gamma, h = v rms:  dx = rms (a - h mean(a h)) + gsum,
//             dgamma = sum over the rows of g h
// The backward pass takes rms from v again, which it has to read anyway, so the forward stores none.
#pragma once
#include "kernels_linear.h"
#include "kernels_norm.h"
#include "mx8.h"

namespace afno {

// ---------------------------------------------------------------- to eight bits and back

// x [M][C] at any address to q, s.  One pass, bound by memory: eight neighbouring values a thread, a load of 16 bytes
// (two in fp32), a block's largest value by two exchanges among its four threads (64,800 x 1,024 bf16: 41 us for 201 MB,
// 4.9 TB/s, a copy's rate; fp32 59 us with one set of inputs, 5.7 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) mx8_pack_kernel(const T* __restrict__ x, Rows8 o, int64_t M, int64_t C) {
  constexpr int UE = Unit<T>::UE, NU = 8 / UE;
  const int64_t per = o.ld / 8, all = M * per;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all; t += (int64_t)gridDim.x * 256) {
    const int64_t m = t / per, c = 8 * (t - m * per);
    union { uint4 u[NU]; T e[8]; } xv;
#pragma unroll
    for (int i = 0; i < NU; ++i) xv.u[i] = Unit<T>::template load<false>(x + m * C + c + UE * i, C - c - UE * i);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)xv.e[i];
    const int byte = block_scale8(v, [](float top) { return lanes_max<4>(top); });
    uint32_t w[2];
    round8(v, byte, w);
    *reinterpret_cast<uint2*>(o.q + m * o.ld + c) = make_uint2(w[0], w[1]);
    if (c % kBlock8 == 0) o.s[m * (o.ld / kBlock8) + c / kBlock8] = (uint8_t)byte;
  }
}

// The values that q, s stand for, eight to a thread, as rows of ldo values (C of them, zeros behind; ALIGNED: ldo a multiple
// of 8 and out 16-byte aligned).  No rounding: the stored values are normal numbers of either type.  Bound by memory
// (64,800 x 1,024 to bf16: 31 to 35 us for 201 MB, 5.7 to 6.5 TB/s, part of the eight bits from the caches; 64,800 x
// 4,096 141 us, 5.7 TB/s; 64,800 x 1,024 to fp32 89 us, 3.8 TB/s, four fifths of it stores).
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) mx8_unpack_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                         int64_t ld, T* __restrict__ out, int64_t ldo, int64_t M) {
  const int64_t per = (ldo + 7) / 8, all = M * per;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all; t += (int64_t)gridDim.x * 256) {
    const int64_t m = t / per, c = 8 * (t - m * per);
    const uint2 w = *reinterpret_cast<const uint2*>(q + m * ld + c);
    const float f = power8(s[m * (ld / kBlock8) + c / kBlock8]);
    T* o = out + m * ldo + c;
    union { uint4 u[8 * sizeof(T) / 16]; T e[8]; uint2 h[2]; float f[8 * sizeof(T) / 4]; } r;
    if constexpr (sizeof(T) == 2) {
      r.h[0] = widen8_bf16(w.x, f);
      r.h[1] = widen8_bf16(w.y, f);
    } else {
      widen8(w.x, f, r.f);
      widen8(w.y, f, r.f + 4);
    }
    if (c + 8 <= ldo) {
      if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(o)[i] = r.u[i];
      } else {
        __builtin_memcpy(o, &r, sizeof(r));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < ldo) o[i] = r.e[i];
    }
  }
}

// ---------------------------------------------------------------- the norm

// Small rows: where the mean square and eps lie below 2^-100, squares of float32 lose digits or vanish (eps 0: a row of
// 1e-23 would divide by 0).  There everything is taken 2^100 times as large, exactly: the largest square is then below
// 2^20 2^100 (2^20 channels), that of the smallest number 2^-98.  The factor 2^100 of 1 / sqrt() stays apart, since
// float32 does not hold it for the smallest rows.  Others keep their steps and their bits; the test costs a scalar branch a row.
constexpr float kSmallRow = 0x1p-100f, kRowUp = 0x1p100f, kRowHalfUp = 0x1p50f;
__device__ __forceinline__ bool small_row(float mean_and_eps) {
  return __builtin_amdgcn_readfirstlane(mean_and_eps < kSmallRow);  // the same in the row's threads
}
// 1 / sqrt(mean(v^2) + eps) of a row; v is 0 behind its channels.  Of a small row v comes back times kRowUp, and the result is
// for that.
template <int W, int NU, int UE>
__device__ __forceinline__ float row_rms(float (&v)[NU][UE], int C, float eps, float* s4, bool* small) {
  auto mean = [&]() {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < UE; ++e) q = __builtin_fmaf(v[i][e], v[i][e], q);
    return row_sum<W>(q, s4) / (float)C;
  };
  float s = mean() + eps;
  *small = small_row(s);
  if (*small) {
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < UE; ++e) v[i][e] *= kRowUp;
    s = mean() + eps * kRowUp * kRowUp;
  }
  return rsqrtf(s);
}

// UE neighbouring values of each of the 32 / UE lanes of a block, to eight bits at channel c of a row
template <int UE>
__device__ __forceinline__ void put8(const Rows8& o, int64_t m, int64_t c, const float (&v)[UE], bool there) {
  const int byte = block_scale8(v, [](float top) { return lanes_max<kBlock8 / UE>(top); });
  uint32_t w[(UE + 3) / 4];
  round8(v, byte, w);
  if (!there) return;
  uint8_t* p = o.q + m * o.ld + c;
  if constexpr (UE == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else if constexpr (UE == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
  else *p = (uint8_t)w[0];
  if (c % kBlock8 == 0) o.s[m * (o.ld / kBlock8) + c / kBlock8] = (uint8_t)byte;
}

// C <= CAP: W waves a row, 4 / W rows a workgroup.  residual, out, sum and o.q may be null.  A row stays in registers
// from its sum to its eight bits, so that everything is read and written once: bound by memory (64,800 x 1,024 bf16 with a
// residual, its sum and eight bits: 91 us for 467 MB, 5.1 TB/s, fp32 149 us with one set of inputs, 5.8 TB/s; one row 2.7 us,
// latency).
template <typename T, bool VEC, int CAP, int W>
__global__ void __launch_bounds__(256) rms_rows(const T* __restrict__ x, const T* __restrict__ residual,
                                                const T* __restrict__ gamma, T* __restrict__ out,
                                                T* __restrict__ sum, Rows8 o, int64_t M, int C, float eps) {
  typedef RowPart<T, VEC, CAP, W> P;
  constexpr int NU = P::NU, UE = P::UE;
  __shared__ float s4[4];
  const int lane = threadIdx.x & (P::NL - 1);
  const int64_t m = (int64_t)blockIdx.x * (4 / W) + threadIdx.x / P::NL;
  if (m >= M) return;  // whole waves; of W = 4 the whole workgroup
  typename P::Raw rx[NU], rr[NU], rg[NU];  // all of the row's loads under way at once
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = UE * (lane + P::NL * i);
    if (c >= C) continue;
    rx[i] = P::raw(x + m * C + c);
    if (residual) rr[i] = P::raw(residual + m * C + c);
    rg[i] = P::raw(gamma + c);
  }
  float v[NU][UE];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = UE * (lane + P::NL * i);
#pragma unroll
    for (int e = 0; e < UE; ++e) v[i][e] = 0.f;
    if (c >= C) continue;
    P::widen(rx[i], v[i]);
    if (residual) {
      float r[UE];
      P::widen(rr[i], r);
#pragma unroll
      for (int e = 0; e < UE; ++e) v[i][e] = (float)Store<T>::to(v[i][e] + r[e]);
    }
    if (sum) P::store(sum + m * C + c, v[i]);
  }
  bool small;
  const float rms = row_rms<W>(v, C, eps, s4, &small);
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = UE * (lane + P::NL * i);
    float y[UE];
#pragma unroll
    for (int e = 0; e < UE; ++e) y[e] = 0.f;
    if (c < C) {
      float ga[UE];
      P::widen(rg[i], ga);
#pragma unroll
      for (int e = 0; e < UE; ++e) y[e] = v[i][e] * rms * ga[e];
      if (out) P::store(out + m * C + c, y);
    }
    if (o.q) put8(o, m, c, y, c < o.ld);
  }
}

// C <= CAP: as norm_rows_backward, rows shared by the grid's workgroups, the next row's loads under way during
// the present one's sums; part [gridDim.x][C].  Bound by memory (64,800 x 1,024 bf16 with gsum: 95 us for 531 MB, 5.6 TB/s,
// fp32 152 us with one set of inputs, part of it from the caches); few odd rows (5,187 x 333 fp32: 9 us) by the latency of
// gamma's and a row's loads and its two sums.
template <typename T, bool VEC, int CAP, int W>
__global__ void __launch_bounds__(256) rms_rows_backward(const T* __restrict__ g, const T* __restrict__ x,
                                                         const T* __restrict__ gamma, const T* __restrict__ gsum,
                                                         T* __restrict__ dx, float* __restrict__ part, int64_t M,
                                                         int C, float eps) {
  typedef RowPart<T, VEC, CAP, W> P;
  constexpr int NU = P::NU, UE = P::UE;
  __shared__ float sums[W == 1 ? CAP : 1];
  __shared__ float s4[4];
  const int lane = threadIdx.x & (P::NL - 1), wave = threadIdx.x / P::NL;
  float dg[NU][UE], ga[NU][UE];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int c = UE * (lane + P::NL * i);
#pragma unroll
    for (int e = 0; e < UE; ++e) dg[i][e] = ga[i][e] = 0.f;
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
#pragma unroll
      for (int e = 0; e < UE; ++e) v[i][e] = a[i][e] = o[i][e] = 0.f;
      if (UE * (lane + P::NL * i) >= C) continue;
      P::widen(rv[i], v[i]);
      P::widen(rg[i], a[i]);
      if (gsum) P::widen(rs[i], o[i]);
    }
    if (m + step < M) fetch(m + step);
    bool small;
    float rms = row_rms<W>(v, C, eps, s4, &small);
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < UE; ++e) {
        v[i][e] *= rms;  // h
        dg[i][e] = __builtin_fmaf(a[i][e], v[i][e], dg[i][e]);
        a[i][e] *= ga[i][e];
        q = __builtin_fmaf(a[i][e], v[i][e], q);
      }
    q = row_sum<W>(q, s4) * inv;
    const float up = small ? kRowHalfUp : 1.f;
    rms *= up;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = UE * (lane + P::NL * i);
      if (c >= C) continue;
#pragma unroll
      for (int e = 0; e < UE; ++e) o[i][e] += rms * (up * (a[i][e] - v[i][e] * q));
      P::store(dx + m * C + c, o[i]);
    }
  }
  if constexpr (W == 4) {
    float* p = part + (int64_t)blockIdx.x * C;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int c = UE * (lane + P::NL * i);
      if (c >= C) continue;
#pragma unroll
      for (int e = 0; e < UE; ++e) p[c + e] = dg[i][e];
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
        for (int e = 0; e < UE; ++e) sums[c + e] = w ? sums[c + e] + dg[i][e] : dg[i][e];
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < C; c += 256) part[(int64_t)blockIdx.x * C + c] = sums[c];
}

// Rows of any width, a workgroup a row, read again for each pass (from the caches): 2,000 x 9,001 bf16
// with a residual, its sum and eight bits 63 us for 127 MB, 2.0 TB/s: value by value, three passes, since a row begins at any
// address and a lane's values of one pass are no longer in registers in the next.
template <typename T>
__global__ void __launch_bounds__(256) rms_wide(const T* __restrict__ x, const T* __restrict__ residual,
                                                const T* __restrict__ gamma, T* __restrict__ out,
                                                T* __restrict__ sum, Rows8 o, int C, float eps) {
  __shared__ float s4[4];
  const int64_t m = blockIdx.x, base = m * C;
  auto at = [&](int c) {
    const float v = ld_f(x + base + c);
    return residual ? (float)Store<T>::to(v + ld_f(residual + base + c)) : v;
  };
  float q = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float v = at(c);
    if (sum) sum[base + c] = Store<T>::to(v);
    q = __builtin_fmaf(v, v, q);
  }
  float mean = group_sum(q, s4) / (float)C + eps, up = 1.f;
  if (small_row(mean)) {
    up = kRowUp;
    q = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float v = at(c) * up;
      q = __builtin_fmaf(v, v, q);
    }
    mean = group_sum(q, s4) / (float)C + eps * up * up;
  }
  const float rms = rsqrtf(mean);
  const int ld = (int)row8(C);  // whole blocks: the 32 lanes of one are in the loop together
  for (int c = threadIdx.x; c < ld; c += 256) {
    float y[1] = {c < C ? at(c) * up * rms * ld_f(gamma + c) : 0.f};
    if (out && c < C) out[base + c] = Store<T>::to(y[0]);
    if (o.q) put8(o, m, c, y, true);
  }
}

// as rms_wide; rms of each row left in stats for rms_columns, of a small row that of the enlarged one with a minus
// sign (2,000 x 9,001 bf16: 45 us, 2.4 TB/s)
template <typename T>
__global__ void __launch_bounds__(256) rms_wide_backward(const T* __restrict__ g, const T* __restrict__ x,
                                                         const T* __restrict__ gamma, const T* __restrict__ gsum,
                                                         T* __restrict__ dx, float* __restrict__ stats, int C,
                                                         float eps) {
  __shared__ float s4[4];
  const int64_t base = (int64_t)blockIdx.x * C;
  float q = 0.f;
  for (int c = threadIdx.x; c < C; c += 256) {
    const float v = ld_f(x + base + c);
    q = __builtin_fmaf(v, v, q);
  }
  float mean = group_sum(q, s4) / (float)C + eps, up = 1.f, half = 1.f;
  if (small_row(mean)) {
    up = kRowUp;
    half = kRowHalfUp;
    q = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float v = ld_f(x + base + c) * up;
      q = __builtin_fmaf(v, v, q);
    }
    mean = group_sum(q, s4) / (float)C + eps * up * up;
  }
  const float rms = rsqrtf(mean);
  if (threadIdx.x == 0) stats[blockIdx.x] = up == 1.f ? rms : -rms;
  float s = 0.f;
  for (int c = threadIdx.x; c < C; c += 256)
    s = __builtin_fmaf(ld_f(g + base + c) * ld_f(gamma + c), ld_f(x + base + c) * up * rms, s);
  s = group_sum(s, s4) / (float)C;
  for (int c = threadIdx.x; c < C; c += 256) {
    float d = half * rms * (half * (ld_f(g + base + c) * ld_f(gamma + c) - ld_f(x + base + c) * up * rms * s));
    if (gsum) d += ld_f(gsum + base + c);
    dx[base + c] = Store<T>::to(d);
  }
}

// dgamma of a chunk of rows (blockIdx.y), a column a thread: part [chunks][C] (2,000 x 9,001 bf16: 18 us, 4.1 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) rms_columns(const T* __restrict__ g, const T* __restrict__ x,
                                                   const float* __restrict__ stats, float* __restrict__ part,
                                                   int64_t M, int C, int64_t rows) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= C) return;
  const int64_t m0 = blockIdx.y * rows, m1 = min(M, m0 + rows);
  float s = 0.f;
  for (int64_t m = m0; m < m1; ++m) {
    const float rms = stats[m], up = rms < 0.f ? kRowUp : 1.f;
    s = __builtin_fmaf(ld_f(g + m * C + c), ld_f(x + m * C + c) * up * fabsf(rms), s);
  }
  part[(int64_t)blockIdx.y * C + c] = s;
}

}  // namespace afno
