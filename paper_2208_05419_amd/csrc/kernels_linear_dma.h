// kernels_linear_dma.h -- the products of kernels_linear.h whose operands are moved straight into the LDS
// (each lane's 16 bytes, without registers or LDS store instructions in between).
//
// k-stages of 128 bytes of a k-major row: 64 bf16, 32 fp32.  The kernels take lda, ldb and, of a row-major
// operand, its rows ma or nb that are multiples of a 16-byte unit (8 bf16, 4 fp32), operands that are
// 16-byte aligned, and kper a multiple of the k-stage; a k-major row has zeros from K to the unit's end.
// M, N and what the epilogue reads and writes are free.  Rows and columns behind an operand's last read
// that one again, into places whose products are not stored; the k's behind the last whole stage come in
// a stage of their own, zeros behind them.
#pragma once
#include "kernels_linear.h"

namespace afno {

// a lane's operand of one k-half of a stage: eight bf16, or four fp32, one to each of four instructions
union DmaOp {
  uint4 u;
  uint2 h[2];
  bf16x8 v;
  float f[4];
};
// acc += the products of a k-half's operands, transposed.  The four fp32 instructions of a tile are spread
// over the tiles, so that none waits for the one before it.
template <typename T, int TM, int TN, int AM>
__device__ __forceinline__ void dma_products(const DmaOp (&fa)[TM], const DmaOp (&fb)[TN], f32x4 (&acc)[AM][TN],
                                             int a0) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b)
        acc[a0 + a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[b].v, fa[a].v, acc[a0 + a][b], 0, 0, 0);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b)
          acc[a0 + a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[b].f[q], fa[a].f[q], acc[a0 + a][b], 0, 0, 0);
  }
}

// each lane's 16 bytes at src to dst + its lane
__device__ __forceinline__ void lds_load16(const char* src, uint4* dst) {
  __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
}

// s_waitcnt operands: at most n loads under way; no LDS operation; neither
constexpr int wait_loads(int n) { return 0x0f70 | (n & 15) | (n >> 4) << 14; }
constexpr int kWaitLds = 0xc07f, kWaitAll = 0x0070;

__device__ __forceinline__ void dma_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// One operand of a workgroup's product: W rows (m or n) of a stage's k's as a slab in the LDS, of which a
// wave takes the WAVE rows from WAVE * its place.  R: row-major.  B: the second operand, whose rows in
// bf16 are dealt to the tiles of 16 so that in the transposed product a lane ends up with eight
// neighbouring columns of every 32 (fp32: four of every 16, without dealing).
//
// k-major: slab rows of 128 bytes, the 16-byte chunk c of row r at place c ^ f(r), so that the rows that
// a pass of ds_read_b128 takes cover the banks once.  Row-major: slab rows k of W values, the 16-byte
// granule c of row k at c ^ f(k).  bf16 takes an operand with two transposing reads, whose pass is half a
// wave, eight rows k of 32 bytes (A) or of four pieces of 8 (B): f moves the rows to other granules, and
// B's odd pieces take the other half of theirs.  fp32 takes it value by value, four rows k of 64 bytes at
// a time, which f spreads.  No bank conflicts by the counters, in any tile of either type.
template <typename T, bool R, bool B, int W, int WAVE, int NT>
struct Slab {
  static constexpr bool H = sizeof(T) == 2;
  static constexpr int UE = 16 / sizeof(T), BK = 128 / sizeof(T);
  static constexpr int CH = 8, U = W * CH, L = U / NT;  // chunks of a k-major row, units, loads a lane
  static_assert(U % NT == 0, "whole loads");
  const T* base;     // the workgroup's first element
  uint32_t at[L];    // this lane's loads, bytes behind a stage's base
  int v[R ? (B && H ? 4 : 1) : 2];  // this lane's operand places, bytes into the slab

  __device__ static __forceinline__ int swizzle(int i) {
    if constexpr (R && H) {
      const int rows = W * 2 >= 256 ? 4 * (i & 3) : 4 * ((i >> 1) & 1);  // (rows of 128 bytes alternate banks)
      return rows | (B ? 1 : 2) * (((i >> 3) ^ (i >> 4)) & 1);
    } else if constexpr (R) {
      return i & 12;
    } else {
      return B && H ? (i & 3) | ((i >> 1) & 4) : i & 7;
    }
  }
  // p, ld: the operand; o, rows: its first row here and how many there are; k: the first k
  __device__ __forceinline__ Slab(const T* p, int64_t ld, int64_t o, int64_t rows, int64_t k, int tid,
                                  int wave) {
    base = p + (R ? k * ld + o : o * ld + k);
    const int64_t left = rows - o;
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int u = tid + NT * j;
      if constexpr (R) {
        const int kk = u / (W / UE), c = (u % (W / UE)) ^ swizzle(kk);
        at[j] = (uint32_t)sizeof(T) * (kk * (uint32_t)ld + (uint32_t)min((int64_t)(UE * c), left - UE));
      } else {
        const int r = u / CH, c = (u % CH) ^ swizzle(r);
        at[j] = (uint32_t)sizeof(T) * ((uint32_t)min((int64_t)r, left - 1) * (uint32_t)ld + UE * c);
      }
    }
    // A, and fp32: row l16 of a tile.  B in bf16: tile b, lane l16 = 4 r + c: column 32 (b / 2) + 8 r +
    // 4 (b % 2) + c; row-major, where odd r take the other half of their granule, 32 (b / 2) + 8 r + 4
    // (b % 2 ^ r % 2) + c.  Of a transposing read, lane 4 r + c gives the address of k = r (+ 4 in the
    // second one) of its 8 gq and of columns 4 c.
    const int lane = tid & 63, l16 = lane & 15, gq = lane >> 4, r4 = l16 >> 2, c4 = l16 & 3;
    if constexpr (R && !H) {
      v[0] = 4 * W * (4 * gq) + 16 * ((WAVE / 4 * wave + r4) ^ swizzle(4 * gq)) + 4 * c4;
    } else if constexpr (R) {
      const int kk = 8 * gq + r4, f = swizzle(kk), g0 = WAVE / 8 * wave;
      if constexpr (B) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
          v[b] = 2 * W * kk + 16 * ((g0 + (WAVE == 64 ? 4 * (b >> 1) : 0) + c4) ^ f) + 8 * ((b ^ c4) & 1);
      } else {
        v[0] = 2 * W * kk + 16 * ((g0 + (c4 >> 1)) ^ f) + 8 * (c4 & 1);
      }
    } else {
      const int r = WAVE * wave + (B && H ? 8 * r4 + c4 : l16);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) v[ks] = 16 * (r * CH + ((4 * ks + gq) ^ swizzle(r)));
    }
  }
  __device__ __forceinline__ const char* stage_base(int64_t k, int64_t ld) const {
    return reinterpret_cast<const char*>(base + (R ? k * ld : k));
  }
  // the loads of the whole stage from k on; d: the slab + 64 * wave
  __device__ __forceinline__ void issue(uint4* d, int64_t k, int64_t ld) const {
    const char* s = stage_base(k, ld);
#pragma unroll
    for (int j = 0; j < L; ++j) lds_load16(s + at[j], d + NT * j);
  }
  // the last `left` k's, fewer than a stage, and zeros
  __device__ __forceinline__ void issue_rest(uint4* d, int64_t k, int64_t ld, int left, int tid) const {
    const char* s = stage_base(k, ld);
#pragma unroll
    for (int j = 0; j < L; ++j) {
      const int u = tid + NT * j, kk = R ? u / (W / UE) : UE * ((u % CH) ^ swizzle(u / CH));
      if (kk < left) lds_load16(s + at[j], d + NT * j);
      else d[NT * j + (tid & 63)] = make_uint4(0, 0, 0, 0);
    }
  }
  // tile t's operand for k-half ks
  __device__ __forceinline__ DmaOp read(const uint4* slab, int ks, int t) const {
    DmaOp o;
    const char* p = reinterpret_cast<const char*>(slab);
    if constexpr (R && !H) {
      p += (v[0] ^ (64 * t)) + 64 * W * ks;
#pragma unroll
      for (int q = 0; q < 4; ++q) o.f[q] = *reinterpret_cast<const float*>(p + 4 * W * q);
    } else if constexpr (R) {
      p += (B ? v[t % 4] : v[0] ^ (32 * t)) + 64 * W * ks;
      o.h[0] = lds_read_tr(p);
      o.h[1] = lds_read_tr(p + 8 * W);
    } else {
      o.u = *reinterpret_cast<const uint4*>(p + v[ks] + (B && H ? 4096 * (t >> 1) + 512 * (t & 1) : 2048 * t));
    }
    return o;
  }
};

// The epilogue of a wave's TM x TN tiles, each wave on its own, without LDS.  This lane has row l16 of
// every 16 and, bf16, columns 8 gq .. + 7 of every 32, fp32, 4 gq .. + 3 of every 16: a store covers 64
// bytes of 16 rows.  m0, n0: the wave's first row and column.
template <typename T, bool BR, int TM, int TN>
__device__ __forceinline__ void dma_store(const GemmArgs<T>& g, const Drop& d, const f32x4 (&acc)[TM][TN],
                                          int64_t m0, int64_t n0, int split, int lane) {
  constexpr int NV = 16 / sizeof(T), PER = NV / 4;
  const int l16 = lane & 15, gq = lane >> 4;
  const bool units = aligned_units<T, NV>(g.e, g.N);
  float bias[TN / PER][NV];  // all loads at once
#pragma unroll
  for (int h = 0; h < TN / PER; ++h) load_bias(g.e, g.N, n0 + NV * gq + 4 * NV * h, bias[h]);
#pragma unroll
  for (int h = 0; h < TN / PER; ++h) {
    const int64_t n = n0 + NV * gq + 4 * NV * h;
    if (n >= g.N) continue;
    const float(&bv)[NV] = bias[h];
#pragma unroll
    for (int a = 0; a < TM; ++a) {
      const int64_t m = m0 + 16 * a + l16;
      __builtin_amdgcn_sched_barrier(0);  // one group's values at a time in registers
      if (m >= g.M) continue;
      float o[NV];
      if constexpr (PER == 2) {
        // row-major B: odd lane groups hold the later four columns in the even tile
        const bool swap = BR && (gq & 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          o[q] = swap ? acc[a][2 * h + 1][q] : acc[a][2 * h][q];
          o[4 + q] = swap ? acc[a][2 * h][q] : acc[a][2 * h + 1][q];
        }
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = acc[a][h][q];
      }
      if (!g.part) {
        finish_some(g.e, d, g.N, m, n, bv, o, units);
        continue;
      }
      float* p = g.part + (split * g.M + m) * g.N + n;
      if (g.N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (n + 4 * i < g.N)
            *reinterpret_cast<float4*>(p + 4 * i) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < NV; ++e)
          if (n + e < g.N) p[e] = o[e];
      }
    }
  }
}

// Workgroup tile 256 x 256, 8 waves as 2 x 4 of 128 x 64, two LDS buffers of 64 KB.
//
// The two waves of a SIMD belong to two groups (waves 0 to 3 and 4 to 7), and the second runs one
// barrier behind the first: while one group reads the operands of its next 16 matrix instructions
// from the LDS, the other has its 16 on the matrix cores, then they change places.  A stage is four such
// turns (k-halves by row halves).  All waves of the one workgroup a CU in step instead: 546 us where this then
// took 496 (64,800 x 1,024 x 4,096).
// The next stage's loads go out in the first two turns and have to be there at the end of the fourth
// read, a barrier before the other group begins to read that stage; the buffer that they fill was read
// for the last time before the barrier ahead of them.
// The 32 x 32 x 16 instruction, whose lanes hold 32 bytes of 32 rows to store: 565 us and 730 us where
// this then took 507 and 567 (64,800 x 4,096 x 1,024 and the other way round).
// Now 446 us = 1.22 PFLOP/s and 545 = 1.00, bound by the matrix cores at the clock that their power leaves and,
// in the wide product, by an epilogue during which one workgroup a CU leaves them idle: GELU and dropout, with the
// value before them stored too, come to about 715.
template <bool AR, bool BR>
__global__ void __launch_bounds__(512) gemm_tile256(GemmArgs<bf16> g) {
  typedef Slab<bf16, AR, false, 256, 128, 512> SA;
  typedef Slab<bf16, BR, true, 256, 64, 512> SB;
  constexpr int BK = 64;
  __shared__ uint4 st0[SA::U + SB::U];
  __shared__ uint4 st1[SA::U + SB::U];
  const TilePlace t((g.M + 256 - 1) / 256, (g.N + 256 - 1) / 256, g.splits);
  if (!t.any) return;
  const int64_t m0 = t.m * 256, n0 = t.n * 256;
  const int64_t k0 = t.split * g.kper, k1 = min(g.K, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
  const int S = (int)((k1 - k0) / BK);  // whole stages
  const SA sa(g.a, g.lda, m0, g.ma, k0, tid, wm);
  const SB sb(g.b, g.ldb, n0, g.nb, k0, tid, wn);

  f32x4 acc[8][4];
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto sync = [&]() {  // everything that this wave has under way, then every wave's
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitAll);
    dma_barrier();
  };
  DmaOp fa[4], fb[4];
  auto stage = [&](const uint4* st, uint4* next, int s) {
    const int64_t kn = (int64_t)min(s + 1, S - 1) * BK;  // behind the last: that again, nobody reads it
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int ks = q >> 1, a0 = 4 * (q & 1);
      if ((q & 1) == 0) {
#pragma unroll
        for (int b = 0; b < 4; ++b) fb[b] = sb.read(st + SA::U, ks, b);
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) fa[a] = sa.read(st, ks, a0 + a);
      if (next && q == 0) sa.issue(next + 64 * wave, kn, g.lda);
      if (next && q == 1) sb.issue(next + SA::U + 64 * wave, kn, g.ldb);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      if (q == 3) __builtin_amdgcn_s_waitcnt(kWaitAll);
      dma_barrier();
      __builtin_amdgcn_s_setprio(1);
      dma_products<bf16>(fa, fb, acc, a0);
      __builtin_amdgcn_s_setprio(0);
      dma_barrier();
    }
  };
  // every wave passes the same number of barriers: the second group one more ahead, the first behind
  if (S) {
    sa.issue(st0 + 64 * wave, 0, g.lda);
    sb.issue(st0 + SA::U + 64 * wave, 0, g.ldb);
  }
  const Drop d(g.e.drop);  // its load of the counter under cover of the first stage's
  if (S) {
    sync();
    if (wave >= 4) dma_barrier();
    int s = 0;
    // no way out inside the loop: with one, the accumulators live in two sets of registers
    for (; s + 1 < S; s += 2) {
      stage(st0, st1, s);
      stage(st1, st0, s + 1);
    }
    if (S & 1) stage(st0, nullptr, s);
    if (wave < 4) dma_barrier();
  }
  if (const int left = (int)(k1 - k0 - (int64_t)S * BK); left > 0) {
    sync();
    sa.issue_rest(st0 + 64 * wave, (int64_t)S * BK, g.lda, left, tid);
    sb.issue_rest(st0 + SA::U + 64 * wave, (int64_t)S * BK, g.ldb, left, tid);
    sync();
    if (wave >= 4) dma_barrier();
    stage(st0, nullptr, 0);
    if (wave < 4) dma_barrier();
  }
  // the surplus loads land before the workgroup's LDS can pass to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(wait_loads(0));
  asm volatile("" ::: "memory");
  dma_store<bf16, BR, 8, 4>(g, d, acc, m0 + 128 * wm, n0 + 64 * wn, t.split, lane);
}

// Workgroup tile TILE x TILE (128 or 64), 4 waves as 2 x 2, fp32 8 as 2 x 4 (two to a SIMD cover each other's
// waits where a CU has one workgroup: 10,368 x 1,536 x 384 126 -> 113 us), for sizes that give the large
// tile too few workgroups.  Stages of 32 KB (16 KB) in two (four) LDS buffers, so that two workgroups share a CU and
// cover each other's waits; the small tile's products are short, so its loads go out three stages
// ahead.  The buffers are separate arrays: the compiler then sees that a buffer being read is not one whose
// loads are under way.
template <typename T>
struct TileWaves {
  static constexpr int N = sizeof(T) == 4 ? 4 : 2, NT = 128 * N;
};
template <typename T, bool AR, bool BR, int TILE>
__global__ void __launch_bounds__((TileWaves<T>::NT)) gemm_tile(GemmArgs<T> g) {
  constexpr int WN = TileWaves<T>::N, NT = TileWaves<T>::NT, WR = TILE / 2, WC = TILE / WN;
  constexpr int TM = WR / 16, TN = WC / 16, NS = TILE == 128 ? 2 : 4;
  typedef Slab<T, AR, false, TILE, WR, NT> SA;
  typedef Slab<T, BR, true, TILE, WC, NT> SB;
  constexpr int BK = SA::BK, U = SA::U + SB::U, L = SA::L + SB::L;
  __shared__ uint4 st0[U];
  __shared__ uint4 st1[U];
  __shared__ uint4 st2[NS == 4 ? U : 1];
  __shared__ uint4 st3[NS == 4 ? U : 1];
  const TilePlace t((g.M + TILE - 1) / TILE, (g.N + TILE - 1) / TILE, g.splits);
  if (!t.any) return;
  const int64_t m0 = t.m * TILE, n0 = t.n * TILE;
  const int64_t k0 = t.split * g.kper, k1 = min(g.K, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int S = (int)((k1 - k0) / BK);  // whole stages
  const SA sa(g.a, g.lda, m0, g.ma, k0, tid, wm);
  const SB sb(g.b, g.ldb, n0, g.nb, k0, tid, wn);

  f32x4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  // stage s (behind the last: that one again, into a buffer nobody reads, so that every wait counts alike)
  auto issue = [&](uint4* st, int s) {
    const int64_t k = (int64_t)min(s, S - 1) * BK;
    sa.issue(st + 64 * wave, k, g.lda);
    sb.issue(st + SA::U + 64 * wave, k, g.ldb);
  };
  auto compute = [&](const uint4* st) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      DmaOp fa[TM], fb[TN];
#pragma unroll
      for (int b = 0; b < TN; ++b) fb[b] = sb.read(st + SA::U, ks, b);
#pragma unroll
      for (int a = 0; a < TM; ++a) fa[a] = sa.read(st, ks, a);
      dma_products<T>(fa, fb, acc, 0);
    }
  };
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
        compute(st0);
        sync();
        issue(st0, s + 2);
        compute(st1);
      }
      sync_all();
      if (S & 1) compute(st0);
    } else {
      for (; s + 3 < S; s += 4) {
        sync();
        issue(st3, s + 3);
        compute(st0);
        sync();
        issue(st0, s + 4);
        compute(st1);
        sync();
        issue(st1, s + 5);
        compute(st2);
        sync();
        issue(st2, s + 6);
        compute(st3);
      }
      sync_all();
      if (S - s > 0) compute(st0);
      if (S - s > 1) compute(st1);
      if (S - s > 2) compute(st2);
    }
  }
  if (const int left = (int)(k1 - k0 - (int64_t)S * BK); left > 0) {
    // a buffer that no wave reads any more: the last that may be is st2, or st0 of two
    uint4* rest = NS == 2 ? st1 : st3;
    if (S) sync_all();
    sa.issue_rest(rest + 64 * wave, (int64_t)S * BK, g.lda, left, tid);
    sb.issue_rest(rest + SA::U + 64 * wave, (int64_t)S * BK, g.ldb, left, tid);
    sync_all();
    compute(rest);
  }
  dma_store<T, BR, TM, TN>(g, d, acc, m0 + WR * wm, n0 + WC * wn, t.split, lane);
}

}  // namespace afno
