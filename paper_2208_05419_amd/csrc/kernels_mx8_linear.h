// kernels_mx8_linear.h -- products of rows in eight bits (mx8.h) with their epilogue:
//   out = drop(act(x w + b)) + residual,   x [M][K], w [N][K] (output-major: both k-major)
// out in the storage type, in eight bits or both, and x w + b in eight bits.
//
// bf16: the matrix cores' scaled instruction, which multiplies 16 x 16 tiles over 128 k's of E4M3 values and
// applies the scales of x and w itself, at twice the rate of bf16.  v_mfma_scale_f32_16x16x128_f8f6f4: lane
// l = 16 gq + l16 gives of row l16 the k's 16 gq .. + 15 and 64 + 16 gq .. + 15 (measured: with a byte of one lane set
// and the scales of all lanes distinct), and the scale of that row's block gq, k's 32 gq .. + 31.  Its sums are in float32
// but for one place: of eight neighbouring k's products the instruction drops what lies below 2^-13 of the
// power of two in the largest (measured: 1 + 2^-13 is kept, 1 + 2^-14 is not, nor any number of them; the unscaled
// instruction does so too), 1.7e-5 of the result in the relative 2-norm at any K, where bfloat16 rounds off 1.7e-3 and
// E4M3 2.6e-2.
//
// fp32, which that would cost seven bits: the values and scales as bfloat16, which holds each of them, on the bf16
// instruction, whose products and sums lose nothing beyond float32's own roundings (6e-8 at 2,048 k's), at half the rate.
#pragma once
#include "kernels_linear_dma.h"
#include "mx8.h"
#include "mx8_rules.h"

namespace afno {

typedef int i32x8 __attribute__((ext_vector_type(8)));
// a lane's operand of a stage: 32 values of a row
union Mx8Op {
  uint4 u[2];
  uint32_t w[8];
  i32x8 v;
};
// a scale byte as mx8_products takes it: the scaled instruction looks at the lowest byte alone
template <typename T>
__device__ __forceinline__ int scale_byte(uint32_t w) {
  return (int)(sizeof(T) == 2 ? w : w & 255);
}
// The accumulators of some row tiles stay in the registers and at the place in the program that they have here: the
// compiler moves products over barriers otherwise, holds their operands for longer, and has too few registers.
template <int TM, int TN>
__device__ __forceinline__ void hold(f32x4 (&acc)[TM][TN], int a0, int n) {
#pragma unroll
  for (int a = 0; a < n; ++a) {
    if constexpr (TN == 4)
      asm volatile("" : "+v"(acc[a0 + a][0]), "+v"(acc[a0 + a][1]), "+v"(acc[a0 + a][2]), "+v"(acc[a0 + a][3]));
    else
      asm volatile("" : "+v"(acc[a0 + a][0]), "+v"(acc[a0 + a][1]));
  }
}
// acc += the products of a stage's operands under their scale bytes, transposed
template <typename T, int TM, int TN, int AM>
__device__ __forceinline__ void mx8_products(const Mx8Op (&fa)[TM], const Mx8Op (&fb)[TN], const int* sa,
                                             const int* sb, f32x4 (&acc)[AM][TN], int a0) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b)
        acc[a0 + a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[b].v, fa[a].v, acc[a0 + a][b], 0, 0, 0,
                                                                          sb[b], 0, sa[a]);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      union Wide { uint2 h[2]; bf16x8 v; } wa[TM], wb[TN];
#pragma unroll
      for (int b = 0; b < TN; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) wb[b].h[i] = widen8_bf16(fb[b].w[2 * s + i], power8(sb[b]));
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int i = 0; i < 2; ++i) wa[a].h[i] = widen8_bf16(fa[a].w[2 * s + i], power8(sa[a]));
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b)
          acc[a0 + a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[b].v, wa[a].v, acc[a0 + a][b], 0, 0, 0);
    }
  }
}

template <typename T>
struct Mx8Args {
  const uint8_t *a, *as, *b, *bs;  // values [M][ld], [N][ld], scales [..][ld / 32]
  int64_t M, N, ld;
  int64_t kper;  // k of one split, a multiple of 128
  int splits;
  float* part;   // [splits][M][N] sums (splits > 1), else null
  Epilogue<T> e; // out may be null; pre is
  Rows8 out8, pre8;
};

// W rows of a stage's 128 k's as a slab in the LDS: rows of 128 bytes, the 16-byte chunk c of row r at place
// c ^ f(r), so that the rows that a pass of ds_read_b128 takes cover the banks once (WIDE: twice).  A wave takes the WAVE rows
// from WAVE * its place.  B: the second operand, whose rows are dealt to the tiles of 16 so that in the
// transposed product a lane ends up with NV = WAVE / 4 neighbouring columns (16, the 16 bytes of a store in eight bits,
// or 8): tile b, lane l16 = 4 r + c has row NV r + 4 b + c.
// WIDE: a lane's two chunks of a row are a block's, 2 gq and 2 gq + 1, and not gq and 4 + gq, so that one scale widens
// both.  Two lane groups' chunks then differ in bit 1 where gq's differ in bit 0, and rows of one parity meet on the same
// banks: 0.43 conflicts an access are counted in fp32.
template <bool B, bool WIDE, int W, int WAVE, int NT>
struct Slab8 {
  static constexpr int CH = 8, U = W * CH, L = U / NT;  // chunks of a row, 16-byte units, loads a lane
  static_assert(U % NT == 0, "whole loads");
  Buf base;  // the workgroup's rows
  // this lane's first load, bytes behind a stage's base, its place in the last row; from load to load
  uint32_t at, last, far;
  int v[2];                // this lane's operand places, bytes into the slab
  const uint8_t* scales;   // of the workgroup's first row
  uint32_t sat, step, most;  // this lane's row of the first tile in them, from tile to tile, the last row

  static constexpr int NV = WAVE / 4;
  __device__ static __forceinline__ int swizzle(int i) { return B ? (i & 3) | (i / (NV / 4) & 4) : i & 7; }
  __device__ __forceinline__ Slab8(const uint8_t* q, const uint8_t* s, int64_t ld, int64_t o, int64_t rows, int tid,
                                   int wave)
      : base(q + o * ld, (uint32_t)(min((int64_t)W, rows - o) * ld)), scales(s + o * (ld / kBlock8)) {
    const int64_t left = rows - o;  // rows behind the last read that one, for products that are not stored
    // (the rows of a lane's loads are NT / CH apart, which the swizzle does not see)
    const int r0 = tid / CH, c = (tid % CH) ^ swizzle(r0);
    at = (uint32_t)r0 * (uint32_t)ld + 16 * c;
    last = (uint32_t)min(left - 1, (int64_t)W) * (uint32_t)ld + 16 * c;
    far = NT / CH * (uint32_t)ld;
    const int lane = tid & 63, l16 = lane & 15, gq = lane >> 4;
    const int r = WAVE * wave + (B ? NV * (l16 >> 2) + (l16 & 3) : l16);
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h] = 16 * (r * CH + ((WIDE ? 2 * gq + h : 4 * h + gq) ^ swizzle(r)));
    const uint32_t sld = (uint32_t)(ld / kBlock8);
    sat = r * sld;
    step = (B ? 4 : 16) * sld;
    most = (uint32_t)min(left - 1, (int64_t)W) * sld;
  }
  // load j of the stage at k
  __device__ __forceinline__ void load(uint4* d, int64_t k, int j) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(base.r, (__attribute__((address_space(3))) void*)(d + NT * j), 16,
                                             (int)min(at + j * far, last), (int)k, 0, 0);
  }
  // the loads of the whole stage from k on; d: the slab + 64 * wave
  __device__ __forceinline__ void issue(uint4* d, int64_t k) const {
#pragma unroll
    for (int j = 0; j < L; ++j) load(d, k, j);
  }
  // the last `left` k's, fewer than a stage, and zeros
  __device__ __forceinline__ void issue_rest(uint4* d, int64_t k, int left, int tid) const {
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int u = tid + NT * j;
      if (16 * ((u % CH) ^ swizzle(u / CH)) < left) load(d, k, j);
      else d[NT * j + (tid & 63)] = make_uint4(0, 0, 0, 0);
    }
  }
  // A stage's operands: the places as they are in this stage alone (opq: one addition each, where the compiler otherwise
  // keeps an address of its own for each tile and buffer in registers across the kernel).
  struct Reader {
    const char *p0, *p1;
    __device__ __forceinline__ Mx8Op operator()(int t) const {
      Mx8Op o;
      o.u[0] = *reinterpret_cast<const uint4*>(p0 + (B ? 512 : 2048) * t);
      o.u[1] = *reinterpret_cast<const uint4*>(p1 + (B ? 512 : 2048) * t);
      return o;
    }
  };
  __device__ __forceinline__ Reader read(const uint4* slab) const {
    const char* p = reinterpret_cast<const char*>(slab);
    return {p + opq(v[0]), p + opq(v[1])};
  }
  // tile t's row of scales; rows behind the last read that one
  __device__ __forceinline__ uint32_t row_of(int t) const { return min(sat + t * step, most); }
  // tile t's scale byte for the stage at k, of which only `left` k's are there; any power for the blocks behind
  // them, where all values are 0
  __device__ __forceinline__ int rest_scale(int64_t k, int t, int gq, int left) const {
    const bool there = 32 * gq < left;
    const int v = scales[row_of(t) + (there ? gq : 0) + (uint32_t)(k / kBlock8)];
    return there ? v : 127;
  }
  // tile t's scale bytes of four stages from k on in one load: lane group gq gets the four blocks of stage gq (of
  // `stages` that are there: of the last one else)
  __device__ __forceinline__ uint32_t four_scales(int64_t k, int t, int gq, int stages) const {
    uint32_t w;
    __builtin_memcpy(&w, scales + row_of(t) + (uint32_t)(k / kBlock8) + 4 * min(gq, stages - 1), 4);
    return w;
  }
};

// four_scales' words of the four lane groups turned round: byte j of lane group gq is block gq of stage j
__device__ __forceinline__ uint32_t turn_scales(uint32_t w, uint32_t sel) {
  const auto h = __builtin_amdgcn_permlane32_swap(w, w, false, false);            // of gq % 2, of gq % 2 + 2
  const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);      // of 0, of 1
  const auto b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);      // of 2, of 3
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[1], b[0], sel), __builtin_amdgcn_perm(a[1], a[0], sel),
                               0x05040100u);
}

// A place in a product's results: row and column, and what lies ahead of it in rows of N values, of ld bytes and of
// scales (products of 64 bits, 32 cycles a wave each: taken once, and from row tile to row tile by addition).
struct Place8 {
  int64_t m, n, at, q, s;
  __device__ __forceinline__ Place8(int64_t m, int64_t n, int64_t N)
      : m(m), n(n), at(m * N + n), q(m * row8(N) + n), s(m * (row8(N) / kBlock8) + n / kBlock8) {}
  __device__ __forceinline__ void down(int rows, int64_t N) {
    m += rows;
    at += rows * N;
    q += rows * row8(N);
    s += rows * (row8(N) / kBlock8);
  }
};

// NV (8 or 16) neighbouring values from a place on, in eight bits; JOIN, which lanes have the rest of the
// block: the next ones or the ones 16 apart.  All lanes of the wave together.  there: the row exists
// (columns behind the last are not stored).
enum { kNeighbours, kRowsApart };
template <int NV, int JOIN>
__device__ __forceinline__ void store8(const Rows8& o, const Place8& p, int64_t N, const float (&z)[NV], bool there) {
  const int64_t n = p.n;
  float v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = z[i];
  if (N % kBlock8) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = n + i < N ? z[i] : 0.f;
  }
  constexpr int LANES = kBlock8 / NV;
  const int byte = block_scale8(v, [](float top) {
    return JOIN == kNeighbours ? lanes_max<LANES>(top) : rows_max<LANES>(top);
  });
  uint32_t w[NV / 4];
  round8(v, byte, w);
  if (!there || n >= o.ld) return;
  uint8_t* q = o.q + p.q;
  if constexpr (NV == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
  if (n % kBlock8 == 0) o.s[p.s] = (uint8_t)byte;
}

// NV values of type T in registers
template <typename T, int NV>
union Some {
  static constexpr int UE = 16 / sizeof(T), NU = NV / UE;
  uint4 u[NU];
  T e[NV];
  // p[0 .. n), 0 behind them, at any address
  __device__ __forceinline__ void load(const T* p, int64_t n) {
#pragma unroll
    for (int i = 0; i < NU; ++i) u[i] = Unit<T>::template load<false>(p + UE * i, n - UE * i);
  }
};

// The epilogue of NV neighbouring values, their biases added; as store8 all lanes of the wave together.  In bf16 the
// short GELU, whose error is below that of the eight-bit instruction (64,800 x 1,024 x 4,096 to eight bits: 422 us, 456 with
// the other one, with dropout and both results 586 and 609; few rows and joined splits take it too, so that a product's
// GELU is the same for any number of rows).  The results in the storage type go out by ordinary stores (392 us; past the
// caches 442).
template <typename T, int NV, int JOIN>
__device__ __forceinline__ void finish8(const Mx8Args<T>& g, const Drop& d, const Place8& p, float (&o)[NV],
                                        bool units) {
  const Epilogue<T>& e = g.e;
  const bool there = p.m < g.M;
  const int64_t n = p.n, at = p.at;
  if (g.pre8.q) store8<NV, JOIN>(g.pre8, p, g.N, o, there);
  if (e.act == kActGelu) {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = sizeof(T) == 2 ? gelu_short(o[i]) : gelu(o[i]);
  } else if (e.act == kActRelu) {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = activate(o[i], kActRelu);
  }
  if (d.threshold) {
#pragma unroll
    for (int h = 0; h < NV / 8; ++h) {
      float(&v)[8] = *reinterpret_cast<float(*)[8]>(o + 8 * h);
      if (g.N % 8 == 0) {
        const uint4 w = d.numbers(((uint64_t)at >> 3) + h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d.apply(v[i], w, i);
      } else {
        d.apply_from(v, (uint64_t)at + 8 * h);
      }
    }
  }
  typedef Some<T, NV> S;
  if (e.residual) {
    S r;
    r.load(e.residual + at, there ? g.N - n : 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] += (float)r.e[i];
  }
  if (e.out) {
    S r;
#pragma unroll
    for (int i = 0; i < NV; ++i) r.e[i] = Store<T>::to(o[i]);
    if (there && n + NV <= g.N) {
      typedef uint32_t Words __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int i = 0; i < S::NU; ++i) {
        if (units)
          *reinterpret_cast<Words*>(e.out + at + S::UE * i) = (Words){r.u[i].x, r.u[i].y, r.u[i].z, r.u[i].w};
        else
          __builtin_memcpy(e.out + at + S::UE * i, &r.u[i], 16);
      }
    } else if (there) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (n + i < g.N) e.out[at + i] = r.e[i];
    }
  }
  if (g.out8.q) store8<NV, JOIN>(g.out8, p, g.N, o, there);
}
template <typename T, int NV>
__device__ __forceinline__ void load_bias8(const Epilogue<T>& e, int64_t N, int64_t n, float (&b)[NV]) {
  Some<T, NV> r;
  r.load(e.bias + n, e.bias ? N - n : 0);
#pragma unroll
  for (int i = 0; i < NV; ++i) b[i] = (float)r.e[i];
}
// whether out takes 16-byte stores
template <typename T>
__device__ __forceinline__ bool whole_units8(const Mx8Args<T>& g) {
  return (uintptr_t)g.e.out % 16 == 0 && g.N % (16 / sizeof(T)) == 0;
}

// NV neighbouring sums of row m from column n on: a split's, or the results.  All lanes of the wave together.
template <typename T, int NV, int JOIN>
__device__ __forceinline__ void mx8_out(const Mx8Args<T>& g, const Drop& d, const Place8& at, int split,
                                        float (&o)[NV], bool units) {
  if (!g.part) {
    finish8<T, NV, JOIN>(g, d, at, o, units);
    return;
  }
  if (at.m >= g.M) return;
  const int64_t n = at.n;
  float* p = g.part + split * g.M * g.N + at.at;
  if (g.N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < NV / 4; ++i)
      if (n + 4 * i < g.N)
        *reinterpret_cast<float4*>(p + 4 * i) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
  } else {
#pragma unroll
    for (int e = 0; e < NV; ++e)
      if (n + e < g.N) p[e] = o[e];
  }
}

// a wave's sums before the first product: the biases of its columns (a split's: 0)
template <typename T, int TM, int TN>
__device__ __forceinline__ void mx8_begin(const Mx8Args<T>& g, f32x4 (&acc)[TM][TN], int64_t n0, int lane) {
  float bias[4 * TN];
#pragma unroll
  for (int i = 0; i < 4 * TN; ++i) bias[i] = 0.f;
  if (g.e.bias && !g.part) load_bias8(g.e, g.N, n0 + 4 * TN * (lane >> 4), bias);
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b)
      acc[a][b] = f32x4{bias[4 * b], bias[4 * b + 1], bias[4 * b + 2], bias[4 * b + 3]};
  hold(acc, 0, TM);
}

// The epilogue of a wave's TM x TN tiles without LDS: this lane has row l16 of every 16 and 4 TN neighbouring
// columns, so that a block of 32 lies in two lanes (four of tiles of 64) and a lane stores 16 bytes.  m0, n0: the wave's
// first row and column.
template <typename T, int TM, int TN>
__device__ __forceinline__ void mx8_store(const Mx8Args<T>& g, const Drop& d, const f32x4 (&acc)[TM][TN],
                                          int64_t m0, int64_t n0, int split, int lane) {
  constexpr int NV = 4 * TN;
  if (n0 >= g.N) return;  // the whole wave's
  const int l16 = lane & 15, gq = lane >> 4;
  const bool units = whole_units8(g);
  Place8 p(m0 + l16, n0 + NV * gq, g.N);
#pragma unroll
  for (int a = 0; a < TM; ++a) {
    __builtin_amdgcn_sched_barrier(0);  // one group's values at a time in registers
    float o[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = acc[a][i / 4][i % 4];
    mx8_out<T, NV, kRowsApart>(g, d, p, split, o, units);
    p.down(16, g.N);
  }
}

// Workgroup tile TILE x TILE (128 or 64), 4 waves as 2 x 2, stages of 128 k's in two (four) LDS buffers of 32 KB
// (16 KB), the next stages' loads under way during the present one's products; two workgroups a CU, one's epilogue
// beside the other's products.  A lane group loads the scales of one stage of four as a word a row, which are turned round
// in registers: with a byte for each stage and row, whose waits come between the stages' loads, 64,800 x 4,096 x 1,024
// took 769 us for 473 in tiles of 128.  Tiles of 128: 10,368 x 1,536 x 384 with GELU 17 us, 720 TFLOP/s, one tile of twelve
// stages on nearly every CU: latency and the one epilogue.  In fp32: 64,800 x 1,024 x 1,024 220 us, 616 TFLOP/s, 16,200 x
// 4,096 x 1,024 157 us, 867 (matrix cores 32 %), bound by the widening of each operand to bfloat16 in every wave that reads
// it, half as often as in tiles of 64 (320 and 211 us), and by the LDS reads for that, whose rows meet on banks (Slab8's WIDE).
// Few rows: 64 x 4,096 x 1,024 in four splits 6.4 us, latency.
template <typename T, int TILE>
__global__ void __launch_bounds__(256, 2) mx8_gemm_tile(Mx8Args<T> g) {
  constexpr int NT = 256, WR = TILE / 2, TM = WR / 16, TN = WR / 16, NS = TILE == 128 ? 2 : 4;
  constexpr bool WIDE = sizeof(T) == 4;
  typedef Slab8<false, WIDE, TILE, WR, NT> SA;
  typedef Slab8<true, WIDE, TILE, WR, NT> SB;
  constexpr int U = SA::U + SB::U, BK = 128;
  __shared__ uint4 st0[U];
  __shared__ uint4 st1[U];
  __shared__ uint4 st2[NS == 4 ? U : 1];
  __shared__ uint4 st3[NS == 4 ? U : 1];
  const TilePlace t((g.M + TILE - 1) / TILE, (g.N + TILE - 1) / TILE, g.splits);
  if (!t.any) return;
  const int64_t m0 = t.m * TILE, n0 = t.n * TILE;
  const int64_t k0 = t.split * g.kper, k1 = min(g.ld, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63, gq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const int S = (int)((k1 - k0) / BK), left = (int)(k1 - k0 - (int64_t)S * BK);  // whole stages, the rest
  const SA sa(g.a, g.as, g.ld, m0, g.M, tid, wm);
  const SB sb(g.b, g.bs, g.ld, n0, g.N, tid, wn);

  f32x4 acc[TM][TN];
  mx8_begin(g, acc, n0 + WR * wn, lane);
  // four stages' scales: those in use, and the next four's words under way
  uint32_t pa[TM], pb[TN], ra[TM], rb[TN];
  const uint32_t sel = (uint32_t)(gq | (4 + gq) << 8);
  auto fetch = [&](int i) {  // of stages i .. i + 3
    const int64_t k = k0 + (int64_t)min(i, S - 1) * BK;
#pragma unroll
    for (int a = 0; a < TM; ++a) ra[a] = sa.four_scales(k, a, gq, max(1, S - i));
#pragma unroll
    for (int b = 0; b < TN; ++b) rb[b] = sb.four_scales(k, b, gq, max(1, S - i));
  };
  auto issue = [&](uint4* st, int i) {
    const int64_t k = k0 + (int64_t)min(i, S - 1) * BK;  // behind the last: that one again, nobody reads it
    sa.issue(st + 64 * wave, k);
    sb.issue(st + SA::U + 64 * wave, k);
  };
  auto products = [&](const uint4* st, const int (&ca)[TM], const int (&cb)[TN]) {
    Mx8Op fa[TM], fb[TN];
    const auto rb = sb.read(st + SA::U);
    const auto ra = sa.read(st);
#pragma unroll
    for (int b = 0; b < TN; ++b) fb[b] = rb(b);
#pragma unroll
    for (int a = 0; a < TM; ++a) fa[a] = ra(a);
    mx8_products<T>(fa, fb, ca, cb, acc, 0);
    hold(acc, 0, TM);
  };
  auto compute = [&](const uint4* st, int i) {  // stage i
    if ((i & 3) == 0) {
#pragma unroll
      for (int a = 0; a < TM; ++a) pa[a] = turn_scales(ra[a], sel);
#pragma unroll
      for (int b = 0; b < TN; ++b) pb[b] = turn_scales(rb[b], sel);
      fetch(i + 4);
    }
    int ca[TM], cb[TN];
#pragma unroll
    for (int a = 0; a < TM; ++a) ca[a] = scale_byte<T>(pa[a] >> 8 * (i & 3));
#pragma unroll
    for (int b = 0; b < TN; ++b) cb[b] = scale_byte<T>(pb[b] >> 8 * (i & 3));
    products(st, ca, cb);
  };
  constexpr int L = SA::L + SB::L;  // loads of a stage, apart from scales
  // this wave's loads of the present stage there (the later ones may be under way), its reads of the last
  // one done, then every wave's
  auto sync = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    __builtin_amdgcn_s_waitcnt(wait_loads((NS - 2) * L));
    dma_barrier();
  };
  auto sync_all = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitAll);
    dma_barrier();
  };
  if (S) {
    fetch(0);
    issue(st0, 0);
    if constexpr (NS == 4) {
      issue(st1, 1);
      issue(st2, 2);
    }
  }
  const Drop d(g.e.drop);
  if (S) {
    int s = 0;
    if constexpr (NS == 2) {
      for (; s + 1 < S; s += 2) {
        sync();
        issue(st1, s + 1);
        compute(st0, s);
        sync();
        issue(st0, s + 2);
        compute(st1, s + 1);
      }
      sync_all();
      if (S & 1) compute(st0, s);
    } else {
      for (; s + 3 < S; s += 4) {
        sync();
        issue(st3, s + 3);
        compute(st0, s);
        sync();
        issue(st0, s + 4);
        compute(st1, s + 1);
        sync();
        issue(st1, s + 5);
        compute(st2, s + 2);
        sync();
        issue(st2, s + 6);
        compute(st3, s + 3);
      }
      sync_all();
      if (S - s > 0) compute(st0, s);
      if (S - s > 1) compute(st1, s + 1);
      if (S - s > 2) compute(st2, s + 2);
    }
  }
  if (left > 0) {
    // a buffer that no wave reads any more: the last that may be is st2, or st0 of two
    uint4* rest = NS == 2 ? st1 : st3;
    if (S) sync_all();
    const int64_t k = k0 + (int64_t)S * BK;
    int ca[TM], cb[TN];
#pragma unroll
    for (int a = 0; a < TM; ++a) ca[a] = sa.rest_scale(k, a, gq, left);
#pragma unroll
    for (int b = 0; b < TN; ++b) cb[b] = sb.rest_scale(k, b, gq, left);
    sa.issue_rest(rest + 64 * wave, k, left, tid);
    sb.issue_rest(rest + SA::U + 64 * wave, k, left, tid);
    sync_all();
    products(rest, ca, cb);
  }
  mx8_store<T, TM, TN>(g, d, acc, m0 + WR * wm, n0 + WR * wn, t.split, lane);
}

// Workgroup tile 256 x 256 in bf16, 8 waves as 2 x 4 of 128 x 64, two LDS buffers of 64 KB, the two groups of waves
// in turn at the LDS and the matrix cores as in gemm_tile256: a stage is four turns of two row tiles by four column tiles.
// The scales of four stages lie in the LDS, 16 bytes to a row, which each thread loads for one row (in registers they
// spill); of the second operand's, four rows that a wave reads lie 256 bytes apart, on the same banks (0.25 conflicts an
// access are counted).  8,192 x 8,192 x 8,192 to eight bits: 433 us, 2,540 TFLOP/s, the matrix cores busy in 59 % of the
// cycles: four turns of 8 products, of which the first waits for twelve reads of 16 bytes and all twelve scales, the others for
// four reads.  64,800 x 4,096 x 1,024 261 us, 2,080 TFLOP/s; 64,800 x 1,024 x 4,096, eight
// stages and an epilogue of 65,536 values, 392 us in bf16, 350 in eight bits, with GELU 420, with dropout and the value
// before GELU in eight bits 591 to 615 (matrix cores 19 %, vector ALUs 44 %): one workgroup a CU, whose epilogue leaves the
// matrix cores idle.  Workgroups that stay, with the next tile's first loads under way during the epilogue: 457 us for 392,
// 638 for 591 (the accumulators and two tiles' places spill); tiles of 256 x 128, two workgroups a CU: 373 for 265.
__global__ void __launch_bounds__(512) mx8_gemm_tile256(Mx8Args<bf16> g) {
  constexpr int BK = 128, TM = 8, TN = 4;
  typedef Slab8<false, false, 256, 128, 512> SA;
  typedef Slab8<true, false, 256, 64, 512> SB;
  __shared__ uint4 st0[SA::U + SB::U];
  __shared__ uint4 st1[SA::U + SB::U];
  __shared__ uint4 scales[2][kScaleRows256];
  const TilePlace t((g.M + 255) / 256, (g.N + 255) / 256, 1);
  if (!t.any) return;
  const int64_t m0 = t.m * 256, n0 = t.n * 256;
  const int tid = threadIdx.x, lane = tid & 63, gq = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
  const int S = (int)(g.ld / BK), left = (int)(g.ld - (int64_t)S * BK);  // whole stages, the rest
  const SA sa(g.a, g.as, g.ld, m0, g.M, tid, wm);
  const SB sb(g.b, g.bs, g.ld, n0, g.N, tid, wn);
  // the row whose scales this thread loads: of a, then of b.  The last four stages' 16 bytes are the row's last 16, with
  // those of fewer stages behind `shift` earlier ones.
  const int blocks = (int)(g.ld / kBlock8);
  const uint8_t* from = wave < 4 ? g.as + m0 * blocks : g.bs + n0 * blocks;
  const uint32_t row = (uint32_t)min((int64_t)(tid & 255), (wave < 4 ? g.M - m0 : g.N - n0) - 1) * (uint32_t)blocks;
  // this wave's places in them
  const int pa = 16 * (128 * wm + l16) + gq, pb = 16 * (256 + 64 * wn + SB::NV * (l16 >> 2) + (l16 & 3)) + gq;

  f32x4 acc[TM][TN];
  mx8_begin(g, acc, n0 + 64 * wn, lane);
  auto sync = [&]() {  // everything that this wave has under way, then every wave's
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitAll);
    dma_barrier();
  };
  // a scale byte; any power for the blocks that a rest has not, where all values are 0
  auto scale = [&](int at, auto rest) {
    const uint8_t v = reinterpret_cast<const uint8_t*>(scales)[at];
    return decltype(rest)::value && 32 * gq >= left ? 127 : (int)v;
  };
  Mx8Op fa[2], fb[TN];
  uint4 next_scales;
  // stage `first` + j, first a multiple of four, from st, the next one into `next` (more: there is one); rest: it has
  // `left` k's alone
  const std::integral_constant<bool, true> yes;
  const std::integral_constant<bool, false> no;
  auto stage = [&](const uint4* st, uint4* next, int first, int j, auto more, auto rest) {
    const int sc = scales_at256(first, j, blocks) - (decltype(rest)::value ? scale_back256(gq, left / kBlock8) : 0);
    const int64_t kn = (int64_t)min(first + j + 1, S - 1) * BK;  // behind the last: that again, nobody reads it
    const auto rb = sb.read(st + SA::U);
    const auto ra = sa.read(st);
    // all scales ahead of the loads into the LDS: the compiler waits for those before it reads an array that it does not
    // see to be another one
    int ca[TM], cb[TN];
#pragma unroll
    for (int b = 0; b < TN; ++b) cb[b] = scale(sc + pb + 16 * 4 * b, rest);
#pragma unroll
    for (int a = 0; a < TM; ++a) ca[a] = scale(sc + pa + 16 * 16 * a, rest);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q == 0) {
#pragma unroll
        for (int b = 0; b < TN; ++b) fb[b] = rb(b);
      }
#pragma unroll
      for (int a = 0; a < 2; ++a) fa[a] = ra(2 * q + a);
      if (decltype(more)::value && q < 2) __builtin_amdgcn_sched_barrier(0);  // the reads first
      if (decltype(more)::value && q == 0) sa.issue(next + 64 * wave, kn);
      if (decltype(more)::value && q == 1) sb.issue(next + SA::U + 64 * wave, kn);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      if (q == 3) __builtin_amdgcn_s_waitcnt(kWaitAll);
      dma_barrier();
      __builtin_amdgcn_s_setprio(1);
      mx8_products<bf16>(fa, fb, ca + 2 * q, cb, acc, 2 * q);
      hold(acc, 2 * q, 2);
      __builtin_amdgcn_s_setprio(0);
      dma_barrier();
    }
  };
  if (S) {
    sa.issue(st0 + 64 * wave, 0);
    sb.issue(st0 + SA::U + 64 * wave, 0);
  }
  if (blocks >= 16) {
    __builtin_memcpy(&next_scales, from + row, 16);
    scales[0][tid] = next_scales;
  } else {
    uint8_t* p = reinterpret_cast<uint8_t*>(&scales[0][tid]);
#pragma unroll 1
    for (int i = 0; i < blocks; ++i) p[i] = from[row + i];
  }
  const Drop d(g.e.drop);  // its load of the counter under cover of the first stage's
  if (S) {
    sync();
    // every wave passes the same number of barriers: the second group one more ahead, the first behind
    if (wave >= 4) dma_barrier();
    int s = 0;
    // no way out or branch inside the loop: with one, the accumulators live in two sets of registers
    for (; s + 3 < S; s += 4) {
      __builtin_memcpy(&next_scales, from + row + next_scales256(s, blocks), 16);
      stage(st0, st1, s, 0, yes, no);
      stage(st1, st0, s, 1, yes, no);
      scales[(s >> 2 & 1) ^ 1][tid] = next_scales;
      stage(st0, st1, s, 2, yes, no);
      stage(st1, st0, s, 3, yes, no);
    }
    if (S & 2) {
      stage(st0, st1, s, 0, yes, no);
      stage(st1, st0, s, 1, yes, no);
    }
    if (S & 1) stage(st0, nullptr, s, S & 2, no, no);
    if (wave < 4) dma_barrier();
  }
  if (left > 0) {
    const int64_t k = (int64_t)S * BK;
    sync();
    sa.issue_rest(st0 + 64 * wave, k, left, tid);
    sb.issue_rest(st0 + SA::U + 64 * wave, k, left, tid);
    sync();
    if (wave >= 4) dma_barrier();
    stage(st0, nullptr, S & ~3, S & 3, no, yes);
    if (wave < 4) dma_barrier();
  }
  // the surplus loads land before the workgroup's LDS can pass to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(wait_loads(0));
  asm volatile("" ::: "memory");
  mx8_store<bf16, TM, TN>(g, d, acc, m0 + 128 * wm, n0 + 64 * wn, 0, lane);
}

// ---------------------------------------------------------------- few rows
//
// Up to 16 rows (serving: single tokens), where the weights' bytes are all the time there is: the same matrix instructions on
// operands straight from memory, each weight read once.  A workgroup takes 32 columns and 16 rows; its 16
// waves take a stage of 128 k's each, as far as there are, and their sums meet in the LDS, added in order.
// 1 x 1,024 x 4,096 with GELU: 3.9 us for 4.3 MB in a graph of a hundred such calls, 1.1 TB/s (fp32 4.2): the latency of two loads one
// after another (a kernel's arguments, then the weights), the sums' meeting and the launch.
template <typename T>
__global__ void __launch_bounds__(64 * kFewRowsWaves) mx8_rows(Mx8Args<T> g) {
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int NW = kFewRowsWaves;
  __shared__ float sums[NW][512];
  const int lane = threadIdx.x & 63, gq = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 32, sld = g.ld / kBlock8;
  // rows behind the last read that one, for products that are not stored; columns dealt as Slab8's
  const int64_t xr = min((int64_t)l16, g.M - 1);
  const uint8_t *x = g.a + xr * g.ld, *xs = g.as + xr * sld, *w[2], *ws[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int64_t r = min(n0 + 8 * (l16 >> 2) + 4 * b + (l16 & 3), g.N - 1);
    w[b] = g.b + r * g.ld;
    ws[b] = g.bs + r * sld;
  }
  auto operand = [&](const uint8_t* p, int64_t k) {
    Mx8Op o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = k + 16 * (WIDE ? 2 * gq + h : 4 * h + gq);
      o.u[h] = make_uint4(0, 0, 0, 0);
      if (at < g.ld) o.u[h] = *reinterpret_cast<const uint4*>(p + at);
    }
    return o;
  };
  auto scale = [&](const uint8_t* p, int64_t k) { return k / kBlock8 + gq < sld ? (int)p[k / kBlock8 + gq] : 127; };
  f32x4 acc[1][2] = {{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}};
  const int64_t k = 128 * wave;
  if (k < g.ld) {
    const Mx8Op fx[1] = {operand(x, k)}, fw[2] = {operand(w[0], k), operand(w[1], k)};
    const int cx[1] = {scale(xs, k)}, cw[2] = {scale(ws[0], k), scale(ws[1], k)};
    mx8_products<T>(fx, fw, cx, cw, acc, 0);
  }
  const int64_t n = n0 + 8 * gq;
  float o[8], bias[8];
  load_bias8(g.e, g.N, n, bias);  // the loads of what is wanted last under cover of the sums
  const Drop d(g.e.drop);
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[wave][64 * i + lane] = acc[0][i / 4][i % 4];
  __syncthreads();
  if (threadIdx.x < 512) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NW; ++j) s += sums[j][threadIdx.x];
    sums[0][threadIdx.x] = s;  // nobody else's column
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = sums[0][64 * i + lane] + bias[i];
  finish8<T, 8, kRowsApart>(g, d, Place8(l16, n, g.N), o, whole_units8(g));
}

// The splits' sums added in order, then the epilogue; eight neighbouring elements a thread, four threads a block
// (64 x 4,096 x 1,024 in four splits: 4.2 us, latency and the launch).
template <typename T>
__global__ void __launch_bounds__(256) mx8_join_splits(Mx8Args<T> g) {
  const int64_t per = row8(g.N) / 8, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = t / per, n = 8 * (t - m * per);
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (m < g.M) {
    const float* p = g.part + m * g.N + n;
    for (int s = 0; s < g.splits; ++s, p += g.M * g.N) {
      if (g.N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (n + 4 * i < g.N) {
            const float4 w = *reinterpret_cast<const float4*>(p + 4 * i);
            v[4 * i] += w.x;
            v[4 * i + 1] += w.y;
            v[4 * i + 2] += w.z;
            v[4 * i + 3] += w.w;
          }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (n + j < g.N) v[j] += p[j];
      }
    }
  }
  const Drop d(g.e.drop);
  float bias[8];
  load_bias8(g.e, g.N, n, bias);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += bias[i];
  finish8<T, 8, kNeighbours>(g, d, Place8(m, n, g.N), v, whole_units8(g));
}

}  // namespace afno
