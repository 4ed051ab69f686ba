// MXFP4 pages: 4-bit values (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with a shared power
// of two (a byte, exponent + 127; 255: NaN) for each block of 32 channels of one token's K or V.
//
// A page of one kv-head is 17 D bytes, four parts one behind the other (t: token of the page, c:
// channel; a byte holds an even channel in its low half and the next one in its high half):
//   K codes   8 D    byte c / 2 of token row t: rows of D / 2 bytes
//   V codes   8 D    [t / 4][c / (D / 16)][t % 4][(c % (D / 16)) / 2]
//   K scales  D / 2  [t][c / 32]
//   V scales  D / 2  [t / 4][c / 32][t % 4]
// The order of V is that of the matrix instruction which contracts over tokens: its operand wants
// four consecutive tokens of a channel in one lane, so a lane's share of a page (four tokens of D / 16
// channels) is one run of bytes, a wave reads the page's V in one load, and no transposition through
// LDS is left.  K's operand wants consecutive channels of a token, which rows give: the page's K is
// one load as well.
#pragma once

#include "ga_internal.hpp"

namespace ga {
namespace {

template <int D>
struct Fp4 {
  static constexpr int PAGE = 17 * D;               // bytes of a page of one kv-head
  static constexpr int V = 8 * D;                   // offsets of the V codes, K scales, V scales
  static constexpr int KS = 16 * D;
  static constexpr int VS = 16 * D + D / 2;
  static constexpr int SL = D / 16;                 // channels of a V slice
  static constexpr int NS = D / 32;                 // scales of a token's K or V
};

// Byte offset in a page of the codes of token t from channel c on (c a multiple of D / 16: the run of
// D / 16 channels is contiguous in K and in V), and of the scale of channel c.
template <int D>
__device__ __forceinline__ int fp4_code(int t, int c, bool v) {
  using F = Fp4<D>;
  return v ? F::V + (((t >> 2) * 16 + c / F::SL) * 4 + (t & 3)) * (F::SL / 2) + (c % F::SL) / 2
           : t * (D / 2) + c / 2;
}
template <int D>
__device__ __forceinline__ int fp4_scale(int t, int c, bool v) {
  using F = Fp4<D>;
  return v ? F::VS + ((t >> 2) * F::NS + c / 32) * 4 + (t & 3) : F::KS + t * F::NS + c / 32;
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The two values of byte B of w, times the power of two in s's exponent, as a pair of bf16: exact (two
// significant bits; bf16 has float32's exponents), and NaN for the scale byte 255.
template <int B>
__device__ __forceinline__ unsigned fp4_pair(unsigned w, float s) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, B));
}

// Scale byte J of w, as the float32 whose exponent it is.
template <int J>
__device__ __forceinline__ float fp4_exp(unsigned w) {
  return __builtin_bit_cast(float, ((w >> (8 * J)) & 0xffu) << 23);
}

// Byte at bit `shift` of w, as the float32 whose exponent it is.  (A wave reads scales as whole words: a
// byte load's register is extended in place, which the compiler waits for where the value is moved.)
__device__ __forceinline__ float fp4_exp_at(unsigned w, unsigned shift) {
  return __builtin_bit_cast(float, __builtin_amdgcn_ubfe(w, shift, 8) << 23);
}


}  // namespace
}  // namespace ga
