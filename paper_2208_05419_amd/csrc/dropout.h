// dropout.h -- which elements dropout keeps, from a counter-based generator, so that no mask is
// ever stored: the forward and the backward pass compute the same one from the same numbers.
//
// Philox4x32 with seven rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers:
// as easy as 1, 2, 3", 2011: the smallest round count of theirs that passes every test of theirs).
// One call gives eight 16-bit numbers, which serve the eight elements 8 i .. 8 i + 7 of a tensor's
// flat index: counter (i low, i high, place low, place high), key the seed.  Sixteen bits rather than
// thirty-two, so that one call serves the 16 bytes of bf16 that a lane stores at once: its 14 products
// of 32 x 32 bits are quarter-rate instructions (about 280 issue cycles of a wave a call).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace afno {

// Element e is kept where its number is at least threshold (0: everything), and scaled then.  place
// is offset + *counter (modulo 2^64; no counter: offset).
struct DropArgs {
  uint64_t seed, offset;
  const uint64_t* counter;
  uint32_t threshold;
  float scale;
};

// a ^ b ^ c in one instruction, which the compiler takes two for
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

struct Drop {
  uint32_t k0, k1, c2, c3, threshold;
  float scale;
  __device__ __forceinline__ explicit Drop(const DropArgs& a)
      : k0((uint32_t)a.seed), k1((uint32_t)(a.seed >> 32)), threshold(a.threshold), scale(a.scale) {
    uint64_t place = a.offset;
    if (a.threshold && a.counter) place += *a.counter;
    // the same in every lane: held once a wave
    c2 = __builtin_amdgcn_readfirstlane((uint32_t)place);
    c3 = __builtin_amdgcn_readfirstlane((uint32_t)(place >> 32));
  }
  // the eight numbers of group i, two to a word, the lower half first
  __device__ __forceinline__ uint4 numbers(uint64_t i) const {
    uint32_t x0 = (uint32_t)i, x1 = (uint32_t)(i >> 32), x2 = c2, x3 = c3, a = k0, b = k1;
#pragma unroll
    for (int r = 0; r < 7; ++r) {
      const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
      x0 = xor3((uint32_t)(q >> 32), x1, a);
      x1 = (uint32_t)q;
      x2 = xor3((uint32_t)(p >> 32), x3, b);
      x3 = (uint32_t)p;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    return make_uint4(x0, x1, x2, x3);
  }
  // a value with number j of a group's words.  The upper half of a word is compared in place: it is at least
  // the threshold exactly where the word is at least the threshold's 65,536 fold.
  __device__ __forceinline__ float apply(float v, const uint4& w, int j) const {
    const uint32_t u = j < 2 ? w.x : (j < 4 ? w.y : (j < 6 ? w.z : w.w));
    const bool keep = j & 1 ? u >= threshold << 16 : (uint16_t)u >= (uint16_t)threshold;
    return keep ? v * scale : 0.f;
  }
  // NV <= 8 neighbouring values from flat index e on, whose numbers may lie in two groups
  template <int NV>
  __device__ __forceinline__ void apply_from(float (&v)[NV], uint64_t e) const {
    const uint4 w0 = numbers(e >> 3), w1 = numbers((e >> 3) + 1);
    const int first = (int)(e & 7);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = first + i;
      v[i] = j < 8 ? apply(v[i], w0, j) : apply(v[i], w1, j - 8);
    }
  }
  __device__ __forceinline__ float apply_at(float v, uint64_t e) const {
    return apply(v, numbers(e >> 3), (int)(e & 7));
  }
};

}  // namespace afno
