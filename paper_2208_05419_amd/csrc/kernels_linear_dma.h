// kernels_linear_dma.h -- the bf16 product of kernels_linear.h for large sizes: operands moved straight
// into the LDS, two groups of waves that take turns on the matrix cores and on the LDS.
#pragma once
#include "kernels_linear.h"

namespace afno {

union DmaOp {
  uint4 u;
  uint2 h[2];
  bf16x8 v;
};
__device__ __forceinline__ f32x4 dma_mma(const DmaOp& a, const DmaOp& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}

// each lane's 16 bytes at src to dst + its lane, without passing through registers
__device__ __forceinline__ void lds_load16(const char* src, uint4* dst) {
  __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
}

// Workgroup tile 256 x 256, 8 waves as 2 x 4 of 128 x 64, k-stages of 64 in two LDS buffers of 64 KB
// (operand A, then B), moved by the direct-to-LDS loads.
//
// The two waves of a SIMD belong to two groups (waves 0 to 3 and 4 to 7), and the second runs one
// barrier behind the first: while one group reads the operands of its next 16 matrix instructions
// from the LDS, the other has its 16 on the matrix cores, then they change places.  A stage is four such
// turns (k-halves by row halves).  All waves in step instead: 546 us against 496 (64,800 x 1,024 x 4,096).
// The next stage's loads go out in the first two turns and have to be there at the end of the fourth
// read, a barrier before the other group begins to read that stage; the buffer that they fill was read
// for the last time before the barrier ahead of them.
//
// k-major operands: slab rows of 128 bytes, the 16-byte chunk c of row r at place c ^ f(r), so that the
// rows that a pass of ds_read_b128 takes cover the banks once.  Row-major ones: slab rows k of 512
// bytes, the granule c (eight columns) of row k at c ^ f(k), and an operand is two transposing reads.  A pass
// of those is half a wave, eight rows k of 32 bytes (A) or four pieces of 8 (B): f moves the rows to
// other granules, and B's odd pieces take the other half of theirs.  No bank conflicts by the
// counters either way.
//
// The products are taken transposed and B's rows are dealt to the tiles so that a lane ends up with
// eight neighbouring columns of a row twice: the epilogue needs no LDS, and a store covers 64 bytes of
// 16 rows.  The 32 x 32 x 16 instruction, whose lanes hold two rows' 32 bytes: 565 us and 730 us where
// this takes 507 and 567 (64,800 x 4,096 x 1,024 and the other way round).
//
// lda, ldb, M (row-major A) or K, and N multiples of 8, all bases 16-byte aligned; kper a multiple of
// 64.  Rows and granules behind an operand's last read that one again, into places whose products are
// not stored; the k's behind the last whole stage come in one of their own, zeros behind them.
template <bool AR, bool BR>
__global__ void __launch_bounds__(512) gemm_tile256(GemmArgs<bf16> g) {
  constexpr int BM = 256, BN = 256, BK = 64, NT = 512, UA = BM * BK / 8, CH = BK / 8, L = UA / NT;
  __shared__ uint4 st0[2 * UA];
  __shared__ uint4 st1[2 * UA];
  const int nbn = (int)((g.N + BN - 1) / BN);
  int64_t mb;
  int nb;
  if (!tile_of((g.M + BM - 1) / BM * nbn, nbn, &mb, &nb)) return;
  const int64_t m0 = mb * BM, n0 = (int64_t)nb * BN;
  const int64_t k0 = blockIdx.y * g.kper, k1 = min(g.K, k0 + g.kper);
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, gq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
  const int S = (int)((k1 - k0) / BK);  // whole stages

  auto fa_of = [](int r) { return r & 7; };
  auto fb_of = [](int r) { return (r & 3) | ((r >> 1) & 4); };
  auto fr_of = [](int k, bool b) { return 4 * (k & 3) | (b ? 1 : 2) * (((k >> 3) ^ (k >> 4)) & 1); };

  // This lane's load j of a stage takes unit u = tid + NT j of an operand's slab: its place in the
  // operand's tile, bytes from a base that the whole workgroup shares, and its first k.
  auto place = [&](auto row_major, auto second, int j) -> uint32_t {
    constexpr bool R = decltype(row_major)::value, B = decltype(second)::value;
    const uint32_t ld = (uint32_t)(B ? g.ldb : g.lda);
    const int64_t left = B ? g.N - n0 : g.M - m0;
    const int u = tid + NT * j;
    if constexpr (R) {
      const int k = u / (BM / 8), c = (u % (BM / 8)) ^ fr_of(k, B);
      return 2 * (k * ld + (uint32_t)min((int64_t)(8 * c), left - 8));
    } else {
      const int r = u / CH, c = (u % CH) ^ (B ? fb_of(r) : fa_of(r));
      return 2 * ((uint32_t)min((int64_t)r, left - 1) * ld + 8 * c);
    }
  };
  auto k_of = [&](auto row_major, auto second, int j) {
    constexpr bool R = decltype(row_major)::value, B = decltype(second)::value;
    const int u = tid + NT * j, r = u / CH;
    if constexpr (R) return u / (BM / 8);
    return 8 * ((u % CH) ^ (B ? fb_of(r) : fa_of(r)));
  };
  constexpr auto ar = std::integral_constant<bool, AR>();
  constexpr auto br = std::integral_constant<bool, BR>();
  constexpr auto isa = std::false_type();
  constexpr auto isb = std::true_type();
  uint32_t pa[L], pb[L];
#pragma unroll
  for (int j = 0; j < L; ++j) {
    pa[j] = place(ar, isa, j);
    pb[j] = place(br, isb, j);
  }
  const bf16* basea = g.a + (AR ? k0 * g.lda + m0 : m0 * g.lda + k0);
  const bf16* baseb = g.b + (BR ? k0 * g.ldb + n0 : n0 * g.ldb + k0);
  // a whole stage's loads of A or B (behind the last stage: that one's again, into a buffer nobody reads)
  auto issue = [&](uint4* st, int s, bool second) {
    const int64_t ka = (int64_t)min(s, S - 1) * BK;
    const char* ba = reinterpret_cast<const char*>(basea + (AR ? ka * g.lda : ka));
    const char* bb = reinterpret_cast<const char*>(baseb + (BR ? ka * g.ldb : ka));
    uint4* d = st + 64 * wave + (second ? UA : 0);
#pragma unroll
    for (int j = 0; j < L; ++j) lds_load16(second ? bb + pb[j] : ba + pa[j], d + NT * j);
  };
  // the last k's, fewer than a stage, and zeros
  auto issue_rest = [&](uint4* st, int left) {
    const int64_t ka = (int64_t)S * BK;
    const char* ba = reinterpret_cast<const char*>(basea + (AR ? ka * g.lda : ka));
    const char* bb = reinterpret_cast<const char*>(baseb + (BR ? ka * g.ldb : ka));
    uint4* d = st + 64 * wave;
    const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < L; ++j) {
      if (k_of(ar, isa, j) < left) lds_load16(ba + pa[j], d + NT * j);
      else d[NT * j + lane] = zero;
      if (k_of(br, isb, j) < left) lds_load16(bb + pb[j], d + UA + NT * j);
      else d[UA + NT * j + lane] = zero;
    }
  };

  f32x4 acc[8][4];
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

  // This lane's operand places, bytes into a stage.  A: row l16 of a tile of 16.  B: tile b, lane l16 = 4 r
  // + c: column 32 (b / 2) + 8 r + 4 (b % 2) + c, or row-major, where odd r take the other half of their
  // granule, 32 (b / 2) + 8 r + 4 (b % 2 ^ r % 2) + c.  Of a transposing read, lane 4 r + c gives
  // the address of k = r (+ 4 in the second one) of its 8 gq and of columns 4 c.
  const int r4 = l16 >> 2, c4 = l16 & 3;
  int va[AR ? 1 : 2], vb[BR ? 4 : 2];
  if constexpr (AR) {
    const int k = 8 * gq + r4;
    va[0] = 512 * k + 16 * ((16 * wm + (c4 >> 1)) ^ fr_of(k, false)) + 8 * (c4 & 1);
  } else {
    const int r = 128 * wm + l16;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) va[ks] = 16 * (r * CH + ((4 * ks + gq) ^ fa_of(r)));
  }
  if constexpr (BR) {
    const int k = 8 * gq + r4;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      vb[b] = 16 * UA + 512 * k + 16 * ((8 * wn + 4 * (b >> 1) + c4) ^ fr_of(k, true)) + 8 * ((b ^ c4) & 1);
  } else {
    const int r = 64 * wn + 8 * r4 + c4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) vb[ks] = 16 * (UA + r * CH + ((4 * ks + gq) ^ fb_of(r)));
  }
  auto read_a = [&](const uint4* st, int ks, int a) {
    DmaOp o;
    const char* p = reinterpret_cast<const char*>(st);
    if constexpr (AR) {
      p += (va[0] ^ (32 * a)) + 16384 * ks;
      o.h[0] = lds_read_tr(p);
      o.h[1] = lds_read_tr(p + 2048);
    } else {
      o.u = *reinterpret_cast<const uint4*>(p + va[ks] + 2048 * a);
    }
    return o;
  };
  auto read_b = [&](const uint4* st, int ks, int b) {
    DmaOp o;
    const char* p = reinterpret_cast<const char*>(st);
    if constexpr (BR) {
      p += vb[b] + 16384 * ks;
      o.h[0] = lds_read_tr(p);
      o.h[1] = lds_read_tr(p + 2048);
    } else {
      o.u = *reinterpret_cast<const uint4*>(p + vb[ks] + 4096 * (b >> 1) + 512 * (b & 1));
    }
    return o;
  };
  auto barrier = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto sync = [&]() {  // everything that this wave has under way, then every wave's
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0), lgkmcnt(0)
    barrier();
  };
  DmaOp fa[4], fb[4];
  auto stage = [&](const uint4* st, uint4* next, int s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int ks = q >> 1, a0 = 4 * (q & 1);
      if ((q & 1) == 0) {
#pragma unroll
        for (int b = 0; b < 4; ++b) fb[b] = read_b(st, ks, b);
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) fa[a] = read_a(st, ks, a0 + a);
      if (next && q < 2) issue(next, s + 1, q == 1);
      __builtin_amdgcn_sched_barrier(0);
      if (q == 3) __builtin_amdgcn_s_waitcnt(0x0070);
      else __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
      barrier();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a0 + a][b] = dma_mma(fb[b], fa[a], acc[a0 + a][b]);
      __builtin_amdgcn_s_setprio(0);
      barrier();
    }
  };
  // every wave passes the same number of barriers: the second group one more ahead, the first behind
  if (S) {
    issue(st0, 0, false);
    issue(st0, 0, true);
    sync();
    if (wave >= 4) barrier();
    int s = 0;
    // no way out inside the loop: with one, the accumulators live in two sets of registers
    for (; s + 1 < S; s += 2) {
      stage(st0, st1, s);
      stage(st1, st0, s + 1);
    }
    if (S & 1) stage(st0, nullptr, s);
    if (wave < 4) barrier();
  }
  if (const int left = (int)(k1 - k0 - (int64_t)S * BK); left > 0) {
    sync();
    issue_rest(st0, left);
    sync();
    if (wave >= 4) barrier();
    stage(st0, nullptr, 0);
    if (wave < 4) barrier();
  }
  // the surplus loads land before the workgroup's LDS can pass to another
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);
  asm volatile("" ::: "memory");

  // each wave on its own: this lane's columns n .. n + 7 of a row for h = 0 and 32 behind them for h = 1
  const Drop d(g.e.drop);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t n = n0 + 64 * wn + 8 * gq + 32 * h;
    if (n >= g.N) continue;
    float bv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bv[e] = g.e.bias && !g.part ? (float)g.e.bias[n + e] : 0.f;
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      const int64_t m = m0 + 128 * wm + 16 * a + l16;
      __builtin_amdgcn_sched_barrier(0);  // one group's values at a time in registers
      if (m >= g.M) continue;
      const int64_t at = m * g.N + n;
      // row-major B: odd lane groups hold the later four columns in the even tile
      const bool swap = BR && (gq & 1);
      float o[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        o[q] = swap ? acc[a][2 * h + 1][q] : acc[a][2 * h][q];
        o[4 + q] = swap ? acc[a][2 * h][q] : acc[a][2 * h + 1][q];
      }
      if (g.part) {
        f32x4* p = reinterpret_cast<f32x4*>(g.part + blockIdx.y * g.M * g.N + at);
        p[0] = f32x4{o[0], o[1], o[2], o[3]};
        p[1] = f32x4{o[4], o[5], o[6], o[7]};
        continue;
      }
      finish8(g.e, d, at, bv, o);
    }
  }
}

}  // namespace afno
