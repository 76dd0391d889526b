// kernels_linear.h -- matrix products with their epilogue, for training around the filter:
//   forward   out = drop(act(x w + b)) + residual      x [M][K], w [K][N]
//   backward  dz = act'(pre) drop(g);  dx = dz w^T,  dw = x^T dz,  db = sum over the rows of dz
// One product D[m][n] = sum_k A(m, k) B(n, k) serves all three; an operand is "k-major" where k is
// its fastest index in memory (x and dz forward and in dx, w in dx) and "row-major" where m or n is
// (w forward, both in dw).
#pragma once
#include "dropout.h"
#include "gelu.h"
#include "kernel_common.h"

namespace afno {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
enum { kActNone = 0, kActRelu = 1, kActGelu = 2 };

// what happens to a product's element (m, n) on its way out
template <typename T>
struct Epilogue {
  const T* bias;      // [N] or null
  const T* residual;  // [M][N] or null
  T* out;             // [M][N]
  T* pre;             // [M][N] or null: the value before the activation
  int act;
  DropArgs drop;
};

template <typename T>
struct GemmArgs {
  const T *a, *b;
  int64_t lda, ldb;   // elements from one row (k for row-major operands) to the next
  int64_t M, N, K;
  int64_t kper;       // k of one split, a multiple of the k-stage; splits = gridDim.y
  float* part;        // [splits][M][N] sums (splits > 1), else null
  Epilogue<T> e;
};

__device__ __forceinline__ float activate(float z, int act) {
  if (act == kActGelu) return gelu(z);
  if (act == kActRelu) return z < 0.f ? 0.f : z;  // NaN stays
  return z;
}
__device__ __forceinline__ float activation_slope(float z, int act) {
  if (act == kActGelu) return gelu_grad(z);
  if (act == kActRelu) return z > 0.f ? 1.f : 0.f;
  return 1.f;
}

// The epilogue of up to `n` neighbouring elements of a row, value by value: any width, any alignment.
template <typename T, int NV>
__device__ __forceinline__ void finish(const Epilogue<T>& e, const Drop& d, int64_t N, int64_t m,
                                       int64_t n, int64_t cols, const float (&v)[NV]) {
  uint64_t group = ~0ull;
  uint4 w = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (n + j >= cols) break;
    const int64_t at = m * N + n + j;
    float z = v[j];
    if (e.bias) z += ld_f(e.bias + n + j);
    if (e.pre) e.pre[at] = Store<T>::to(z);
    z = activate(z, e.act);
    if (d.threshold) {
      if (((uint64_t)at >> 3) != group) w = d.numbers(group = (uint64_t)at >> 3);
      z = d.apply(z, w, (int)(at & 7));
    }
    if (e.residual) z += ld_f(e.residual + at);
    e.out[at] = Store<T>::to(z);
  }
}

// The same of eight neighbouring elements of bf16 from `at` on, a multiple of 8, with their biases; out,
// pre and residual 16-byte aligned.  Streamed once: non-temporal, so that they do not push the
// products' operands out of the caches.
__device__ __forceinline__ void finish8(const Epilogue<bf16>& e, const Drop& d, int64_t at,
                                        const float (&bias)[8], float (&o)[8]) {
  auto store = [&](bf16* p) {
    const u32x4 w = {cvt_pk(o[0], o[1]), cvt_pk(o[2], o[3]), cvt_pk(o[4], o[5]), cvt_pk(o[6], o[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p + at));
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] += bias[i];
  if (e.pre) store(e.pre);
  if (e.act == kActGelu) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = gelu(o[i]);
  } else if (e.act == kActRelu) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = activate(o[i], kActRelu);
  }
  if (d.threshold) {
    const uint4 w = d.numbers((uint64_t)at >> 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = d.apply(o[i], w, i);
  }
  if (e.residual) {
    const u32x4 r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(e.residual + at));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      o[i] += i % 2 ? __uint_as_float(r[i / 2] & 0xffff0000u) : __uint_as_float(r[i / 2] << 16);
  }
  store(e.out);
}

// workgroup -> (tile row, tile column): workgroup g runs on XCD g % 8, and the workgroups of one XCD
// take neighbouring tiles, column tiles first, so that a row tile's operand stays in that XCD's L2
__device__ __forceinline__ bool tile_of(int64_t ntile, int nbn, int64_t* mb, int* nb) {
  const int64_t per = (ntile + 7) / 8, g = blockIdx.x, t = (g & 7) * per + (g >> 3);
  if ((g >> 3) >= per || t >= ntile) return false;
  *mb = t / nbn;
  *nb = (int)(t - *mb * nbn);
  return true;
}

// One 16-byte unit (UE elements along the operand's fastest index) in registers.
template <typename T> struct Unit {
  static constexpr int UE = 16 / sizeof(T);
  // elements p[0 .. n), the rest 0; n <= 0: none.  VEC: p is 16-byte aligned and n is never between
  template <bool VEC>
  __device__ static uint4 load(const T* p, int64_t n) {
    union { uint4 u; T e[UE]; } r;
    r.u = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
      if (n > 0) r.u = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < UE; ++i)
        if (i < n) r.e[i] = p[i];
    }
    return r.u;
  }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ds_read_b64_tr_b16: of every 16 lanes, lane 4 r + c gives the address of columns 4 c .. 4 c + 3 of
// row r, and lane i gets column i of rows 0 .. 3 (four 16-bit values).
__device__ __forceinline__ uint2 lds_read_tr(const void* p) {
  union { s16x4 s; uint2 u; } r;
  r.s = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4*)(__attribute__((address_space(3))) void*)const_cast<void*>(p));
  return r.u;
}

// ---------------------------------------------------------------- any size, any alignment
//
// Register-staged product: 256 threads, workgroup tile BM x BN, 2 x 2 waves, k-stages of 32 through
// two LDS stages, the next stage's loads in flight during the present one's matrix instructions.
// k-major operands lie in the LDS as [row][32 + pad] and row-major ones as [32][rows + pad], as they
// come: the fp32 instruction takes single values from either, the bf16 one its eight k's from a row or
// through the transposing LDS read.  The products are taken transposed (D's rows are n), so that a
// lane holds four neighbouring columns of one row.
// VEC: lda, ldb multiples of a 16-byte unit and both bases 16-byte aligned.
template <typename T, bool AR, bool BR, int BM, int BN>
struct RegGeo {
  static constexpr int BK = 32, UE = Unit<T>::UE, PAD = UE;
  static constexpr int LA = AR ? BM + PAD : BK + PAD, LB = BR ? BN + PAD : BK + PAD;  // LDS strides
  static constexpr int SA = (AR ? BK : BM) * LA, SB = (BR ? BK : BN) * LB;            // one stage
  static constexpr int UA = BM * BK / UE / 256, UB = BN * BK / UE / 256;              // units a thread
  static constexpr int kBytes = 2 * (SA + SB) * (int)sizeof(T);
};

template <typename T, bool AR, bool BR, int BM, int BN, bool VEC>
__global__ void __launch_bounds__(256) gemm_reg(GemmArgs<T> g) {
  typedef RegGeo<T, AR, BR, BM, BN> G;
  constexpr int BK = G::BK, UE = G::UE, TM = BM / 32, TN = BN / 32;
  extern __shared__ uint4 reg_smem[];
  T* S = reinterpret_cast<T*>(reg_smem);
  const int nbn = (int)((g.N + BN - 1) / BN);
  int64_t mb;
  int nb;
  if (!tile_of((g.M + BM - 1) / BM * nbn, nbn, &mb, &nb)) return;
  const int64_t m0 = mb * BM, n0 = (int64_t)nb * BN;
  const int64_t k0 = blockIdx.y * g.kper, k1 = min(g.K, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, gq = lane >> 4;
  const int wm = (tid >> 6) >> 1, wn = (tid >> 6) & 1;

  // unit u of a stage: k-major: row u / (BK / UE), k UE (u % ..); row-major: k u / (rows / UE), ..
  auto load = [&](auto row_major, const T* p, int64_t ld, int64_t r0, int64_t rows, int bm, int u,
                  int64_t kb) {
    constexpr bool R = decltype(row_major)::value;
    if constexpr (R) {
      const int per = bm / UE, kk = u / per, r = UE * (u - kk * per);
      const int64_t k = kb + kk;
      return Unit<T>::template load<VEC>(p + k * ld + r0 + r, k < k1 ? rows - r0 - r : 0);
    } else {
      constexpr int per = BK / UE;
      const int r = u / per, kk = UE * (u - r * per);
      const int64_t k = kb + kk;
      return Unit<T>::template load<VEC>(p + (r0 + r) * ld + k, r0 + r < rows ? k1 - k : 0);
    }
  };
  auto slot = [&](auto row_major, int bm, int ldl, int u) {
    constexpr bool R = decltype(row_major)::value;
    const int per = (R ? bm : BK) / UE, r = u / per;
    return r * ldl + UE * (u - r * per);
  };
  constexpr auto ar = std::integral_constant<bool, AR>();
  constexpr auto br = std::integral_constant<bool, BR>();
  uint4 ra[G::UA], rb[G::UB];
  auto fetch = [&](int64_t kb) {
#pragma unroll
    for (int j = 0; j < G::UA; ++j) ra[j] = load(ar, g.a, g.lda, m0, g.M, BM, tid + 256 * j, kb);
#pragma unroll
    for (int j = 0; j < G::UB; ++j) rb[j] = load(br, g.b, g.ldb, n0, g.N, BN, tid + 256 * j, kb);
  };
  auto put = [&](int st) {
    T* sa = S + st * (G::SA + G::SB);
#pragma unroll
    for (int j = 0; j < G::UA; ++j)
      *reinterpret_cast<uint4*>(sa + slot(ar, BM, G::LA, tid + 256 * j)) = ra[j];
#pragma unroll
    for (int j = 0; j < G::UB; ++j)
      *reinterpret_cast<uint4*>(sa + G::SA + slot(br, BN, G::LB, tid + 256 * j)) = rb[j];
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

  // operand of tile t (16 rows from `row`) at k-step kk: bf16 k 8 gq .. + 7 of 32, fp32 k 4 gq .. + 3
  // of 16 (one to each of four instructions)
  auto frag = [&](auto row_major, const T* s, int ldl, int row, int kk) {
    constexpr bool R = decltype(row_major)::value;
    union { uint4 u; uint2 h[2]; float f[4]; } r;
    if constexpr (!R) {
      r.u = *reinterpret_cast<const uint4*>(s + (row + l16) * ldl + kk + UE * gq);
    } else if constexpr (sizeof(T) == 2) {
      const T* p = s + (kk + 8 * gq + (l16 >> 2)) * ldl + row + 4 * (l16 & 3);
      r.h[0] = lds_read_tr(p);
      r.h[1] = lds_read_tr(p + 4 * ldl);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) r.f[q] = ld_f(s + (kk + 4 * gq + q) * ldl + row + l16);
    }
    return r.u;
  };

  const int64_t stages = k1 > k0 ? (k1 - k0 + BK - 1) / BK : 0;
  if (stages) {
    fetch(k0);
    put(0);
  }
  __syncthreads();
  for (int64_t s = 0; s < stages; ++s) {
    const int st = (int)(s & 1);
    if (s + 1 < stages) fetch(k0 + (s + 1) * BK);
    const T* sa = S + st * (G::SA + G::SB);
    const T* sb = sa + G::SA;
    constexpr int KS = sizeof(T) == 2 ? 32 : 16;
#pragma unroll
    for (int kk = 0; kk < BK; kk += KS) {
      uint4 fa[TM], fb[TN];
#pragma unroll
      for (int a = 0; a < TM; ++a) fa[a] = frag(ar, sa, G::LA, BM / 2 * wm + 16 * a, kk);
#pragma unroll
      for (int b = 0; b < TN; ++b) fb[b] = frag(br, sb, G::LB, BN / 2 * wn + 16 * b, kk);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
          for (int b = 0; b < TN; ++b) {
            union { uint4 u; bf16x8 v; } x, y;
            x.u = fb[b];
            y.u = fa[a];
            acc[a][b] = Mma<bf16>::mma(x.v, y.v, acc[a][b]);
          }
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b) {
              V16 x, y;
              x.u = fb[b];
              y.u = fa[a];
              acc[a][b] = Mma<float>::mma(x.f[q], y.f[q], acc[a][b]);
            }
      }
    }
    if (s + 1 < stages) put(st ^ 1);
    __syncthreads();
  }

  const Drop d(g.e.drop);
#pragma unroll
  for (int a = 0; a < TM; ++a) {
    const int64_t m = m0 + BM / 2 * wm + 16 * a + l16;
    if (m >= g.M) continue;
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      const int64_t n = n0 + BN / 2 * wn + 16 * b + 4 * gq;
      float v[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
      if (g.part) {
        float* p = g.part + (blockIdx.y * g.M + m) * g.N + n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n + j < g.N) p[j] = v[j];
      } else {
        finish<T, 4>(g.e, d, g.N, m, n, g.N, v);
      }
    }
  }
}

// The splits' sums added in order, then the epilogue; four neighbouring elements a thread.
template <typename T>
__global__ void __launch_bounds__(256) join_splits(const float* __restrict__ part, int splits,
                                                   int64_t M, int64_t N, Epilogue<T> e) {
  const int64_t per = (N + 3) / 4, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= M * per) return;
  const int64_t m = t / per, n = 4 * (t - m * per);
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  const float* p = part + m * N + n;
  if (N % 4 == 0) {  // 16-byte aligned: the workspace is
    for (int s = 0; s < splits; ++s, p += M * N) {
      const float4 w = *reinterpret_cast<const float4*>(p);
      v[0] += w.x;
      v[1] += w.y;
      v[2] += w.z;
      v[3] += w.w;
    }
  } else {
    for (int s = 0; s < splits; ++s, p += M * N) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < N) v[j] += p[j];
    }
  }
  const Drop d(e.drop);
  finish<T, 4>(e, d, N, m, n, N, v);
}

// ---------------------------------------------------------------- dz and the bias gradient
//
// dz = act'(pre) drop(g), rounded to T for the matrix cores (the one rounding of the backward pass
// before its results'), and the sums over chunks of rows of the unrounded dz, part [chunks][N].  A
// workgroup takes the rows of one chunk (blockIdx.y) and 256 columns: VEC (N a multiple of 8, all
// bases 16-byte aligned) 32 threads of eight columns by eight rows at a time, whose sums meet in the
// LDS; else a column a thread.  dz or part may be null.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dz_kernel(const T* __restrict__ g, const T* __restrict__ pre,
                                                 T* __restrict__ dz, float* __restrict__ part,
                                                 int64_t M, int64_t N, int64_t rows, int act,
                                                 DropArgs da) {
  const int64_t m0 = blockIdx.y * rows, m1 = min(M, m0 + rows);
  const Drop d(da);
  if constexpr (!VEC) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    float s = 0.f;
    for (int64_t m = m0; m < m1; ++m) {
      const int64_t at = m * N + n;
      float v = ld_f(g + at);
      if (d.threshold) v = d.apply_at(v, (uint64_t)at);
      if (act) v *= activation_slope(ld_f(pre + at), act);
      if (dz) dz[at] = Store<T>::to(v);
      s += v;
    }
    if (part) part[blockIdx.y * N + n] = s;
  } else {
    __shared__ float sums[8][256];
    constexpr int UE = Unit<T>::UE, NU = 8 / UE;
    const int c = 8 * (threadIdx.x & 31), r = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 256 + c;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (n < N) {
      for (int64_t m = m0 + r; m < m1; m += 8) {
        const int64_t at = m * N + n;
        union { uint4 u[NU]; T e[8]; } gv, pv, ov;
#pragma unroll
        for (int i = 0; i < NU; ++i) gv.u[i] = reinterpret_cast<const uint4*>(g + at)[i];
        if (act) {
#pragma unroll
          for (int i = 0; i < NU; ++i) pv.u[i] = reinterpret_cast<const uint4*>(pre + at)[i];
        }
        uint4 w = make_uint4(0, 0, 0, 0);
        if (d.threshold) w = d.numbers((uint64_t)at >> 3);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = (float)gv.e[j];
          if (d.threshold) v = d.apply(v, w, j);
          if (act) v *= activation_slope((float)pv.e[j], act);
          s[j] += v;
          ov.e[j] = Store<T>::to(v);
        }
        if (dz) {
#pragma unroll
          for (int i = 0; i < NU; ++i) reinterpret_cast<uint4*>(dz + at)[i] = ov.u[i];
        }
      }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[r][c + j] = s[j];
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col < N) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
      part[blockIdx.y * N + col] = t;
    }
  }
}

// The sums over `chunks` of part[chunk][n], n < N, in an order that does not change: 16 threads of a
// column take every sixteenth chunk, then their sums are added.  16 columns a workgroup.  Columns from
// `first` on go to out2.
template <typename T>
__global__ void __launch_bounds__(256) join_columns(const float* __restrict__ part, int chunks,
                                                    int64_t N, int64_t first, T* __restrict__ out,
                                                    T* __restrict__ out2) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t n = (int64_t)blockIdx.x * 16 + c;
  float s = 0.f;
  if (n < N)
    for (int i = r; i < chunks; i += 16) s += part[(int64_t)i * N + n];
  sums[r][c] = s;
  __syncthreads();
  if (r == 0 && n < N) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += sums[i][c];
    if (n < first)
      out[n] = Store<T>::to(t);
    else
      out2[n - first] = Store<T>::to(t);
  }
}

// ---------------------------------------------------------------- dropout of a tensor
//
// out = drop(x) + residual (null: none) over n elements, eight to a thread.  VEC: all bases 16-byte
// aligned.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const T* __restrict__ x,
                                                      const T* __restrict__ residual,
                                                      T* __restrict__ out, int64_t n, DropArgs da) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, at = 8 * i;
  if (at >= n) return;
  const Drop d(da);
  uint4 w = make_uint4(0, 0, 0, 0);
  if (d.threshold) w = d.numbers((uint64_t)i);
  constexpr int NU = 8 / Unit<T>::UE;
  union { uint4 u[NU]; T e[8]; } xv, rv, ov;
  if (VEC && at + 8 <= n) {
#pragma unroll
    for (int j = 0; j < NU; ++j) xv.u[j] = reinterpret_cast<const uint4*>(x + at)[j];
    if (residual) {
#pragma unroll
      for (int j = 0; j < NU; ++j) rv.u[j] = reinterpret_cast<const uint4*>(residual + at)[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v = (float)xv.e[j];
      if (d.threshold) v = d.apply(v, w, j);
      if (residual) v += (float)rv.e[j];
      ov.e[j] = Store<T>::to(v);
    }
#pragma unroll
    for (int j = 0; j < NU; ++j) reinterpret_cast<uint4*>(out + at)[j] = ov.u[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (at + j >= n) break;
      float v = ld_f(x + at + j);
      if (d.threshold) v = d.apply(v, w, j);
      if (residual) v += ld_f(residual + at + j);
      out[at + j] = Store<T>::to(v);
    }
  }
}

}  // namespace afno
