// mx8.h -- rows of channels in eight bits ("mx8"): E4M3 values (four exponent bits, three of mantissa, bias 7,
// largest 448, no infinity, NaN 0x7f and 0xff) and one power of two for every 32 neighbouring channels of a row,
// the layout of the Open Compute Project's microscaling formats, which the matrix cores' scaled instructions take.
//
//   values [M][ld], ld = C rounded up to 32, zeros behind the C;  scales [M][ld / 32], bytes s + 127
//   value = E4M3 value 2^s;  s: the smallest with which no finite value of the block is above 448, kept in
//   -117 .. 119
// The bounds of s: from 2^-117 up every value that can be stored, 2^(s - 9) and more in size, is a normal bfloat16 (and
// float32) number, so that reading never rounds; up to 2^119 the largest, 448 2^119, is finite: a block with a
// value above that has it at 448 2^119.  A NaN or an infinity becomes NaN and says nothing about s.
#pragma once
#include "kernel_common.h"

namespace afno {

constexpr int kBlock8 = 32;  // channels to a scale
constexpr int kLeast8 = -117, kMost8 = 119;
__host__ __device__ __forceinline__ int64_t row8(int64_t C) { return (C + kBlock8 - 1) / kBlock8 * kBlock8; }

// rows in eight bits: ld = row8(channels) bytes and ld / 32 scales a row; q null: none
struct Rows8 {
  uint8_t *q, *s;
  int64_t ld;
};

// the largest size of N values and `top`; a NaN says nothing
template <int N>
__device__ __forceinline__ float largest8(const float (&v)[N], float top) {
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]));
  return top;
}
// the same of the finite ones, where an infinity is among them
template <int N>
__device__ __forceinline__ float largest_finite8(const float (&v)[N]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float a = fabsf(v[i]);
    top = fmaxf(top, a < __builtin_inff() ? a : 0.f);
  }
  return top;
}
// the scale byte for values of which `top` is the largest in size
__device__ __forceinline__ int scale8(float top) {
  const uint32_t u = __float_as_uint(top);
  // 2^e (1 + f): s = e - 8, one more where 1 + f is above 1.75
  const int s = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(s, kLeast8), kMost8) + 127;
}
// 2^s of a scale byte
__device__ __forceinline__ float power8(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// N values (one, or a multiple of four) divided by 2^s and rounded to E4M3, to nearest, ties to even; the instruction
// makes NaN of what is NaN, infinite or too large
template <int N>
__device__ __forceinline__ void round8(const float (&z)[N], int byte, uint32_t (&w)[(N + 3) / 4]) {
  static_assert(N == 1 || N % 4 == 0, "whole words, or one value");
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  const float scale = power8(byte);
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = z[i];
  if (byte == kMost8 + 127) {  // values above 448 2^119
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (fabsf(v[i]) < __builtin_inff()) v[i] = __builtin_amdgcn_fmed3f(v[i], -448.f * 0x1p119f, 448.f * 0x1p119f);
  }
  union { s16x2 h; uint32_t u; } x;
  x.u = 0;
  if constexpr (N == 1) {
    x.h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x.h, v[0], 0.f, scale, false);
    w[0] = x.u;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      x.h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x.h, v[4 * i], v[4 * i + 1], scale, false);
      x.h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x.h, v[4 * i + 2], v[4 * i + 3], scale, true);
      w[i] = x.u;
    }
  }
}

// four values of a word, times 2^s
__device__ __forceinline__ void widen8(uint32_t w, float scale, float* v) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
  v[0] = a[0];
  v[1] = a[1];
  v[2] = b[0];
  v[3] = b[1];
}
// the same as bfloat16, which holds each of them
__device__ __forceinline__ uint2 widen8_bf16(uint32_t w, float scale) {
  union { bf16x2v v[2]; uint2 u; } r;
  r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
  r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  return r.u;
}

template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)));
}
// the largest over N neighbouring lanes (N aligned lanes, a power of two up to 32), in each of them
template <int N>
__device__ __forceinline__ float lanes_max(float v) {
  if constexpr (N >= 2) v = dpp_max<0xb1>(v);   // quad_perm 1 0 3 2
  if constexpr (N >= 4) v = dpp_max<0x4e>(v);   // quad_perm 2 3 0 1
  if constexpr (N >= 8) v = dpp_max<0x141>(v);  // row_half_mirror: the other four of eight
  if constexpr (N >= 16) v = dpp_max<0x140>(v); // row_mirror: the other eight of sixteen
  if constexpr (N >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
  return v;
}
// the largest over lanes l and l + 32
__device__ __forceinline__ float halves_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
// the largest over N lanes 16 apart: l and l + 16 of every 32, or l, l + 16, l + 32 and l + 48
template <int N>
__device__ __forceinline__ float rows_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  return N == 4 ? halves_max(v) : v;
}

// The scale byte of a block whose values lie in several lanes, N in each, JOIN the largest over them: all lanes of
// the wave together.  Infinities are looked for only in a wave that has one.
template <int N, typename F>
__device__ __forceinline__ int block_scale8(const float (&v)[N], F join) {
  float top = join(largest8(v, 0.f));
  if (__builtin_amdgcn_ballot_w64(top == __builtin_inff())) top = join(largest_finite8(v));
  return scale8(top);
}

}  // namespace afno
