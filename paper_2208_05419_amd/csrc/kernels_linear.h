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
  int64_t ma, nb;     // rows of a and b that are there to be read: M and N, or rounded up to a unit
  int64_t kper;       // k of one split, a multiple of the k-stage
  int splits;
  float* part;        // [splits][M][N] sums (splits > 1), else null
  Epilogue<T> e;
};

__device__ __forceinline__ float activate(float z, int act) {
  if (act == kActGelu) return gelu(z);
  if (act == kActRelu) return z < 0.f ? 0.f : z;  // NaN stays
  return z;
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

// The same of NV = 4 or 8 neighbouring elements from `at` on, all there, with their biases.  ALIGNED: at a
// multiple of NV and out, pre and residual aligned to NV elements; streamed once: non-temporal, so that
// they do not push the products' operands out of the caches (64,800 x 1,024 x 4,096: 554 us, 644 with ordinary
// stores).  Else the same loads and stores at any address.
template <typename T, int NV, bool ALIGNED>
__device__ __forceinline__ void finish_unit(const Epilogue<T>& e, const Drop& d, int64_t at,
                                            const float (&bias)[NV], float (&o)[NV]) {
  typedef uint32_t Words __attribute__((ext_vector_type(NV * sizeof(T) / 4)));
  constexpr int NW = NV * sizeof(T) / 4;
  auto store = [&](T* p) {
    Words w;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      if constexpr (sizeof(T) == 2) w[i] = cvt_pk(o[2 * i], o[2 * i + 1]);
      else w[i] = __float_as_uint(o[i]);
    }
    if constexpr (ALIGNED) __builtin_nontemporal_store(w, reinterpret_cast<Words*>(p + at));
    else __builtin_memcpy(p + at, &w, sizeof(w));
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) o[i] += bias[i];
  if (e.pre) store(e.pre);
  if (e.act == kActGelu) {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = gelu(o[i]);
  } else if (e.act == kActRelu) {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = activate(o[i], kActRelu);
  }
  if (d.threshold) {
    if constexpr (ALIGNED) {
      uint4 w = d.numbers((uint64_t)at >> 3);
      if (NV == 4 && (at & 4)) w = make_uint4(w.z, w.w, w.z, w.w);
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = d.apply(o[i], w, i);
    } else {
      d.apply_from(o, (uint64_t)at);
    }
  }
  if (e.residual) {
    Words r;
    if constexpr (ALIGNED) r = __builtin_nontemporal_load(reinterpret_cast<const Words*>(e.residual + at));
    else __builtin_memcpy(&r, e.residual + at, sizeof(r));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (sizeof(T) == 2)
        o[i] += i % 2 ? __uint_as_float(r[i / 2] & 0xffff0000u) : __uint_as_float(r[i / 2] << 16);
      else
        o[i] += __uint_as_float(r[i]);
    }
  }
  store(e.out);
}
// whether NV neighbouring elements can go through it aligned
template <typename T, int NV>
__host__ __device__ __forceinline__ bool aligned_units(const Epilogue<T>& e, int64_t N) {
  const uintptr_t all = (uintptr_t)e.out | (uintptr_t)e.pre | (uintptr_t)e.residual;
  return N % NV == 0 && all % (NV * sizeof(T)) == 0;
}
// up to NV neighbouring elements of row m from column n on; `units`: aligned_units
template <typename T, int NV>
__device__ __forceinline__ void finish_some(const Epilogue<T>& e, const Drop& d, int64_t N, int64_t m, int64_t n,
                                            const float (&bias)[NV], float (&v)[NV], bool units) {
  if (units) {
    finish_unit<T, NV, true>(e, d, m * N + n, bias, v);
  } else if (n + NV <= N) {
    finish_unit<T, NV, false>(e, d, m * N + n, bias, v);
  } else {
    finish<T, NV>(e, d, N, m, n, N, v);  // takes the bias itself
  }
}
template <typename T, int NV>
__device__ __forceinline__ void load_bias(const Epilogue<T>& e, int64_t N, int64_t n, float (&b)[NV]) {
  union { uint32_t w[NV * sizeof(T) / 4]; T v[NV]; } u = {};
  if (e.bias && n + NV <= N) {
    __builtin_memcpy(u.w, e.bias + n, sizeof(u));  // one load, at any address
  } else if (e.bias) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (n + j < N) u.v[j] = e.bias[n + j];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) b[j] = (float)u.v[j];
}

// Workgroup -> split, tile row and tile column, of 8 ceil(splits tiles / 8) workgroups: workgroup g runs on XCD
// g % 8, and the workgroups of one XCD take neighbouring ones, column tiles first, then rows, then splits, so
// that a row tile's operand stays in that XCD's L2 and no XCD has more than its eighth (252 workgroups dealt by
// tile alone left one XCD with 7 and the others with 35 for 32 CUs: 192 us where 108).  Of eight
// column tiles or more, and of four rounds of the chip or more, rows in groups of eight, a group's columns one
// after another: the 32 tiles that an XCD has under way then read four column tiles' operand and not all of it, which
// the L2 does not hold (64,800 x 1,024 x 4,096 with GELU and dropout, 4,064 tiles, x not in the caches: 795 us by
// rows, 740 by groups of four, 715 of eight; but 4,096 x 1,024 x 4,096, 256 tiles: 35.6 by rows, 37.5 by eight, and
// 2,001 x 1,001 x 999, 512 tiles: 20.6 and 21.9).
struct TilePlace {
  int64_t m, n;
  int split;
  bool any;
  __device__ __forceinline__ TilePlace(int64_t rows, int64_t cols, int splits) {
    // (a launch has fewer than 2^31 workgroups)
    const uint32_t nc = (uint32_t)cols, tiles = (uint32_t)rows * nc, all = tiles * (uint32_t)splits;
    const uint32_t per = (all + 7) / 8, g = blockIdx.x, t = (g & 7) * per + (g >> 3);
    any = (g >> 3) < per && t < all;
    const uint32_t s = t / tiles, i = t - s * tiles, r = i / nc;
    split = (int)s;
    const uint32_t h0 = nc >= 8 && all >= 1024 ? 8 : 1, first = r / h0 * h0, in = i - first * nc;
    const uint32_t h = min(h0, (uint32_t)rows - first);
    n = in / h;
    m = first + (in - in / h * h);
  }
};

// One 16-byte unit (UE elements along the operand's fastest index) in registers.
template <typename T> struct Unit {
  static constexpr int UE = 16 / sizeof(T);
  // elements p[0 .. n), the rest 0; n <= 0: none.  VEC: p is 16-byte aligned and n is never between.
  // Else one load too where all are there: global memory takes it at any address.
  template <bool VEC>
  __device__ static uint4 load(const T* p, int64_t n) {
    union { uint4 u; T e[UE]; } r;
    r.u = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
      if (n > 0) r.u = *reinterpret_cast<const uint4*>(p);
    } else if (n >= UE) {
      __builtin_memcpy(&r.u, p, 16);
    } else if (n > 0) {
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
// Register-staged product: 256 threads, workgroup tile BM x BN, 2 x 2 waves, k-stages of 64 bf16 or 32
// fp32 through two LDS stages, the next stage's loads in flight during the present one's matrix instructions.
// k-major operands lie in the LDS as [row][k + pad] and row-major ones as [k][rows + pad], as they
// come: the fp32 instruction takes single values from either, the bf16 one its eight k's from a row or
// through the transposing LDS read.  The products are taken transposed (D's rows are n), so that a
// lane holds four neighbouring columns of one row.
template <typename T, bool AR, bool BR, int BM, int BN>
struct RegGeo {
  static constexpr int BK = 128 / sizeof(T), UE = Unit<T>::UE, PAD = UE;
  static constexpr int LA = AR ? BM + PAD : BK + PAD, LB = BR ? BN + PAD : BK + PAD;  // LDS strides
  static constexpr int SA = (AR ? BK : BM) * LA, SB = (BR ? BK : BN) * LB;            // one stage
  static constexpr int UA = BM * BK / UE / 256, UB = BN * BK / UE / 256;              // units a thread
  static constexpr int kBytes = 2 * (SA + SB) * (int)sizeof(T);
};

template <typename T, bool AR, bool BR, int BM, int BN>
__global__ void __launch_bounds__(256) gemm_reg(GemmArgs<T> g) {
  typedef RegGeo<T, AR, BR, BM, BN> G;
  constexpr int BK = G::BK, UE = G::UE, TM = BM / 32, TN = BN / 32;
  __shared__ uint4 smem[G::kBytes / 16];
  T* S = reinterpret_cast<T*>(smem);
  const TilePlace t((g.M + BM - 1) / BM, (g.N + BN - 1) / BN, g.splits);
  if (!t.any) return;
  const int64_t m0 = t.m * BM, n0 = t.n * BN;
  const int64_t k0 = t.split * g.kper, k1 = min(g.K, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, gq = lane >> 4;
  const int wm = (tid >> 6) >> 1, wn = (tid >> 6) & 1;

  // unit u of a stage: k-major: row u / (BK / UE), k UE (u % ..); row-major: k u / (rows / UE), ..
  auto load = [&](auto row_major, const T* p, int64_t ld, int64_t r0, int64_t rows, int bm, int u,
                  int64_t kb) {
    constexpr bool R = decltype(row_major)::value;
    if constexpr (R) {
      const int per = bm / UE, kk = u / per, r = UE * (u - kk * per);
      const int64_t k = kb + kk;
      return Unit<T>::template load<false>(p + k * ld + r0 + r, k < k1 ? rows - r0 - r : 0);
    } else {
      constexpr int per = BK / UE;
      const int r = u / per, kk = UE * (u - r * per);
      const int64_t k = kb + kk;
      return Unit<T>::template load<false>(p + (r0 + r) * ld + k, r0 + r < rows ? k1 - k : 0);
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
  const bool units = aligned_units<T, 4>(g.e, g.N);
#pragma unroll
  for (int a = 0; a < TM; ++a) {
    const int64_t m = m0 + BM / 2 * wm + 16 * a + l16;
    if (m >= g.M) continue;
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      const int64_t n = n0 + BN / 2 * wn + 16 * b + 4 * gq;
      if (n >= g.N) continue;
      float v[4] = {acc[a][b][0], acc[a][b][1], acc[a][b][2], acc[a][b][3]};
      if (g.part) {
        float* p = g.part + (t.split * g.M + m) * g.N + n;
        if (g.N % 4 == 0) {
          *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (n + j < g.N) p[j] = v[j];
        }
      } else {
        float bv[4];
        load_bias(g.e, g.N, n, bv);
        finish_some(g.e, d, g.N, m, n, bv, v, units);
      }
    }
  }
}

// ---------------------------------------------------------------- few rows
//
// D = x w of a few rows (serving: single tokens), where the weights' bytes are all the time there is:
// each is read once per MR rows, on the vector ALUs, straight from memory.  A workgroup takes 32
// columns and MR rows (blockIdx.y); its 16 waves take k's in turn, a load of a wave 32 columns of 16
// (fp32 8) k's.  Each lane sums its columns, the 16 lanes of a DPP row add theirs in registers, and the
// 64 DPP rows' sums meet in the LDS, added in order.  w row-major, at any address and of any width.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int kRowsCols = 32;  // 64 bytes of a row of bf16 weights: 16 columns, 1,024 of 4,096 k's: 9.7 us, 32: 6.6
template <typename T, int MR>
__global__ void __launch_bounds__(1024) linear_rows(GemmArgs<T> g) {
  constexpr int UE = Unit<T>::UE, COLS = kRowsCols, LC = COLS / UE, KR = 64 / LC, PF = 4;
  __shared__ float sums[64][MR * COLS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t n = (int64_t)blockIdx.x * COLS + UE * (lane % LC), m0 = (int64_t)blockIdx.y * MR;
  float acc[MR][UE];
#pragma unroll
  for (int r = 0; r < MR; ++r)
#pragma unroll
    for (int e = 0; e < UE; ++e) acc[r][e] = 0.f;
  const T* w = g.b + n;
  const int64_t here = g.N - n;  // columns of this lane's that are there
  const T* x[MR];
#pragma unroll
  for (int r = 0; r < MR; ++r) x[r] = g.a + min(m0 + r, g.M - 1) * g.lda;
  // PF loads of the weights under way in each lane
  for (int64_t k0 = wave * KR + lane / LC; k0 < g.K; k0 += 16 * KR * PF) {
    union { uint4 u; T e[UE]; } wv[PF];
    float xv[PF][MR];
#pragma unroll
    for (int i = 0; i < PF; ++i) {
      const int64_t k = k0 + 16 * KR * i;
      wv[i].u = Unit<T>::template load<false>(w + k * g.ldb, k < g.K ? here : 0);
#pragma unroll
      for (int r = 0; r < MR; ++r) xv[i][r] = k < g.K ? ld_f(x[r] + k) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < PF; ++i)
#pragma unroll
      for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int e = 0; e < UE; ++e) acc[r][e] = __builtin_fmaf(xv[i][r], (float)wv[i].e[e], acc[r][e]);
  }
#pragma unroll
  for (int r = 0; r < MR; ++r)
#pragma unroll
    for (int e = 0; e < UE; ++e) {
      float v = acc[r][e];
      v = dpp_add<0x128>(v);                      // row_ror:8
      if constexpr (LC <= 4) v = dpp_add<0x124>(v);  // row_ror:4
      if ((lane & 15) < LC) sums[tid >> 4][r * COLS + UE * (lane & 15) + e] = v;
    }
  __syncthreads();
  const Drop d(g.e.drop);
  for (int i = tid; i < MR * COLS; i += 1024) {
    const int64_t m = m0 + i / COLS, c = (int64_t)blockIdx.x * COLS + i % COLS;
    if (m >= g.M || c >= g.N) continue;
    float v[1] = {0.f};
    for (int j = 0; j < 64; ++j) v[0] += sums[j][i];
    finish<T, 1>(g.e, d, g.N, m, c, g.N, v);
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
  float bv[4];
  load_bias(e, N, n, bv);
  finish_some(e, d, N, m, n, bv, v, aligned_units<T, 4>(e, N));
}

// ---------------------------------------------------------------- dz and the bias gradient
//
// dz = act'(pre) drop(g), rounded to T for the matrix cores (the one rounding of the backward pass
// before its results'; in bf16 it takes dx and dw from 0.0017 to 0.0023 off float64 in the relative 2-norm, where
// dz in two bf16 terms would double the products, 880 of 1,220 us at 64,800 x 1,024 x 4,096), rows of ldz values, zeros behind the N of dz; and the sums over chunks of rows of the
// unrounded dz, part [chunks][N].  A workgroup takes the rows of one chunk (blockIdx.y) and 256 columns:
// 32 threads of eight columns by eight rows at a time, whose sums meet in the LDS.  VEC: N a multiple of 8,
// g and pre 16-byte aligned.  dz (16-byte aligned, ldz a multiple of 8) or part may be null.
// Bound by the vector ALUs and memory alike: 64,800 x 4,096 bf16 with GELU and dropout 327 us for 1.6 GB
// (4.9 TB/s), 243 without the store of dz, 92 for the sums of g alone; the activation chosen once for eight
// values, 337 with the choice at each value.  The next rows' loads under way meanwhile: 330, not kept.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dz_kernel(const T* __restrict__ g, const T* __restrict__ pre,
                                                 T* __restrict__ dz, int64_t ldz, float* __restrict__ part,
                                                 int64_t M, int64_t N, int64_t rows, int act, DropArgs da) {
  __shared__ float sums[8][256];
  constexpr int UE = Unit<T>::UE, NU = 8 / UE;
  const int64_t m0 = blockIdx.y * rows, m1 = min(M, m0 + rows);
  const Drop d(da);
  const int c = 8 * (threadIdx.x & 31), r = threadIdx.x >> 5;
  const int64_t n = (int64_t)blockIdx.x * 256 + c;
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (n < N) {
    for (int64_t m = m0 + r; m < m1; m += 8) {
      const int64_t at = m * N + n;
      union { uint4 u[NU]; T e[8]; } gv, pv, ov;
#pragma unroll
      for (int i = 0; i < NU; ++i) gv.u[i] = Unit<T>::template load<VEC>(g + at + UE * i, N - n - UE * i);
      if (act) {
#pragma unroll
        for (int i = 0; i < NU; ++i) pv.u[i] = Unit<T>::template load<VEC>(pre + at + UE * i, N - n - UE * i);
      }
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (float)gv.e[j];
      if (d.threshold) {
        if constexpr (VEC) {
          const uint4 w = d.numbers((uint64_t)at >> 3);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = d.apply(v[j], w, j);
        } else {
          d.apply_from(v, (uint64_t)at);
        }
      }
      if (act == kActGelu) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= gelu_grad((float)pv.e[j]);
      } else if (act == kActRelu) {  // selected: an infinity at a unit that is off is no NaN
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)pv.e[j] > 0.f ? v[j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!VEC && n + j >= N) v[j] = 0.f;
        s[j] += v[j];
        ov.e[j] = Store<T>::to(v[j]);
      }
      if (dz) {
#pragma unroll
        for (int i = 0; i < NU; ++i) reinterpret_cast<uint4*>(dz + m * ldz + n)[i] = ov.u[i];
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

// Rows of `cols` values at any address copied to rows of ld (a multiple of a 16-byte unit), zeros behind
// them, so that the direct-to-LDS kernels can take them: two arrays in one launch, the units of the first,
// then the second's (rows2 = 0: none).
template <typename T>
struct PackArgs {
  const T* src;
  T* dst;
  int64_t rows, cols, ld;
};
template <typename T>
__global__ void __launch_bounds__(256) pack_rows(PackArgs<T> a, PackArgs<T> b) {
  constexpr int UE = Unit<T>::UE;
  const int64_t na = a.rows * (a.ld / UE), all = na + b.rows * (b.ld / UE);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const PackArgs<T>& p = i < na ? a : b;
    const int64_t u = i < na ? i : i - na, per = p.ld / UE, r = u / per, c = UE * (u - r * per);
    const uint4 w = Unit<T>::template load<false>(p.src + r * p.cols + c, p.cols - c);
    *reinterpret_cast<uint4*>(p.dst + r * p.ld + c) = w;
  }
}

// The sums over `chunks` of part[chunk][n], n < N, in an order that does not change: 64 threads of a
// column take every 64th chunk, then their sums are added.  16 columns a workgroup.  Columns from `first` on
// go to out2.  Eight chunks' loads are under way at a time: one after another they took longer than the
// kernel that made them (512 chunks of 666 columns: 17 of 29 us).
template <typename T>
__global__ void __launch_bounds__(1024) join_columns(const float* __restrict__ part, int chunks,
                                                     int64_t N, int64_t first, T* __restrict__ out,
                                                     T* __restrict__ out2) {
  __shared__ float sums[64][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t n = (int64_t)blockIdx.x * 16 + c;
  float s = 0.f;
  if (n < N) {
    for (int i = r; i < chunks; i += 512) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = i + 64 * j < chunks ? part[(int64_t)(i + 64 * j) * N + n] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
  }
  sums[r][c] = s;
  __syncthreads();
  if (r == 0 && n < N) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += sums[i][c];
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
