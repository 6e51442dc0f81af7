// Rows held in 8 or 4 bits: 32 consecutive dimensions of a row share a scale 2^e.
//
// With a the largest magnitude of a block, e is the smallest exponent with a <= M 2^e,
// M = 7 (e2m1, largest code 6) or 464 (e4m3, largest code 448): the point half a step
// above the largest code, so that no element is off by more than half a step of its
// binade. Codes are rounded to nearest even by the conversion instructions, which scale by
// 2^e exactly. e is held with a bias of 127 in a byte. Its least value keeps every code
// but 0 a normal bf16 number; magnitudes are cut at what the largest e can hold. A block
// with an element that is not finite has byte 255: the conversions make each of its
// values NaN. A decoded value has four significant bits at most and is a bf16 number as
// it stands, so that matrix products of it are the products of the cache.
//
// Two dimensions of one row are a pair, 4-bit codes in one byte (the even one low), 8-bit
// codes in two. K is [row][pair] with the scales [row][block] behind, V is [pair][row]
// with [block][row] behind: a conversion takes a pair and one scale, so that both layouts
// are decoded a pair an instruction, and V comes out as the operand that attention needs
// after a swap of halves.
#ifndef LDR_MX_H
#define LDR_MX_H

#include "serve_internal.h"

namespace ldr {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

template <int BITS> struct Mx;
template <> struct Mx<4> {
  static constexpr float kLimit = 0.875f, kTop = 0x1.8p127f;   // M = 0.875 * 2^3
  static constexpr int kLimitExp = 3, kLowest = -125;
};
template <> struct Mx<8> {
  static constexpr float kLimit = 0.90625f, kTop = 0x1.ep127f;  // M = 0.90625 * 2^9
  static constexpr int kLimitExp = 9, kLowest = -117;
};

// Scale byte B of a word, as the conversions take it: the exponent of a float, whose other
// bits they do not look at (all 256 exponents with several mantissas and signs give the same
// value of every code, and 255 gives NaN).
template <int B> __device__ inline float mx_scale(uint32_t w) {
  static_assert(B >= 0 && B < 4, "a byte of the word");
  return __uint_as_float(B == 3 ? w >> 1 : w << (23 - 8 * B));
}

// A pair of bf16, the even dimension low: pair I of the words at w.
template <int BITS, int I> __device__ inline uint32_t mx_pair(const uint32_t* w, float scale) {
  if constexpr (BITS == 4)
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[I / 4], scale, I % 4));
  else
    return __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[I / 2], scale, I % 2 == 1));
}

// Eight dimensions of a row (BITS / 4 words) under one scale.
template <int BITS> __device__ inline void mx_eight(const uint32_t* w, float scale, uint32_t* out) {
  out[0] = mx_pair<BITS, 0>(w, scale);
  out[1] = mx_pair<BITS, 1>(w, scale);
  out[2] = mx_pair<BITS, 2>(w, scale);
  out[3] = mx_pair<BITS, 3>(w, scale);
}

// Eight rows of a pair of dimensions (BITS / 2 words), their scales the bytes of two words:
// pairs as they come, one a row.
template <int BITS>
__device__ inline void mx_rows8(const uint32_t* w, uint32_t s0, uint32_t s1, uint32_t* out) {
  out[0] = mx_pair<BITS, 0>(w, mx_scale<0>(s0));
  out[1] = mx_pair<BITS, 1>(w, mx_scale<1>(s0));
  out[2] = mx_pair<BITS, 2>(w, mx_scale<2>(s0));
  out[3] = mx_pair<BITS, 3>(w, mx_scale<3>(s0));
  out[4] = mx_pair<BITS, 4>(w, mx_scale<0>(s1));
  out[5] = mx_pair<BITS, 5>(w, mx_scale<1>(s1));
  out[6] = mx_pair<BITS, 6>(w, mx_scale<2>(s1));
  out[7] = mx_pair<BITS, 7>(w, mx_scale<3>(s1));
}
// The same, turned: eight rows of the even dimension, eight of the odd one.
template <int BITS>
__device__ inline void mx_turned8(const uint32_t* w, uint32_t s0, uint32_t s1, uint32_t* even,
                                  uint32_t* odd) {
  uint32_t x[8];
  mx_rows8<BITS>(w, s0, s1, x);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    even[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x05040100u);
    odd[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x07060302u);
  }
}

// The exponent for a block's largest magnitude (finite, at most kTop).
template <int BITS> __device__ inline int mx_exponent(float a) {
  // frexp of 0 is 0, 0: below the lowest
  const int e = (int)__builtin_amdgcn_frexp_expf(a) - Mx<BITS>::kLimitExp +
                (__builtin_amdgcn_frexp_mantf(a) > Mx<BITS>::kLimit);
  return max(a == 0.f ? Mx<BITS>::kLowest : e, Mx<BITS>::kLowest);
}

// One code, where few are needed: its value.
template <int BITS> __device__ inline float mx_value(uint32_t code, uint32_t scale) {
  uint32_t w[2] = {code, 0};
  return __uint_as_float(mx_pair<BITS, 0>(w, mx_scale<0>(scale)) << 16);
}

}  // namespace
}  // namespace ldr
#endif
