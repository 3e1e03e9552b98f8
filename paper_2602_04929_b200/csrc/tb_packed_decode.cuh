// Packed codes to bf16 integers c - z, exact for |c - z| <= 256 (with the zero-point's second piece, where it has one).
#pragma once

#include "tb_common.cuh"

namespace tb {

// Field of NB bits from bit POS of the words on.
template <int POS, int NB, int N>
__device__ __forceinline__ unsigned field(const unsigned (&w)[N]) {
  constexpr int i = POS >> 5, s = POS & 31;
  unsigned v;
  if constexpr (s + NB <= 32)
    v = w[i] >> s;
  else
    v = __funnelshift_r(w[i], w[i + 1], s);
  if constexpr (NB < 32) v &= (1u << NB) - 1u;
  return v;
}

__device__ __forceinline__ unsigned bf2(__nv_bfloat162 v) { return *reinterpret_cast<const unsigned*>(&v); }
__device__ __forceinline__ __nv_bfloat162 bf2(unsigned v) { return *reinterpret_cast<const __nv_bfloat162*>(&v); }

// (v & mask) | bits in one instruction: with two constants the compiler makes two of it
__device__ __forceinline__ unsigned masked(unsigned v, unsigned mask, unsigned bits) {
  unsigned o;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(o) : "r"(v), "r"(mask), "r"(bits));
  return o;
}
// A zero-point as the decoders take it: 2^23 + z in float for eight bits, else -(128 + z) in two pieces of bf16, the first (in the upper
// half) truncated: what a code and the first piece come to so is no larger than c - z, and exact where that is.  The second piece is 0 for
// -384 <= z <= 128, which a zero-point among the codes always is, so it is added where a warp meets one that is not.
__device__ __forceinline__ unsigned zero_word(int z, int bits) {
  if (bits == 8) return __float_as_uint((float)z + 8388608.0f);
  const float v = -128.0f - (float)z, first = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  return __byte_perm(bf2(__float2bfloat162_rn(v - first)), __float_as_uint(v), 0x7610);
}
template <int BITS>
__device__ __forceinline__ unsigned zero_first(unsigned word) {  // twice, as decode8 takes it
  return BITS == 8 ? word : __byte_perm(word, 0, 0x3232);
}
template <int BITS>
__device__ __forceinline__ unsigned zero_second(unsigned word) {  // twice
  return BITS == 8 ? 0u : __byte_perm(word, 0, 0x1010);
}
template <int BITS>
__device__ __forceinline__ bool has_second(unsigned words) {  // of one word, or of several or-ed together
  return BITS < 8 && (words & 0xffffu) != 0;
}
// Codes C0 .. C0 + 7 of a lane's words as four pairs of bf16 holding c - z.  A code placed in the low mantissa bits of 128.0
// is 128 + c (up to seven bits), and 128 + z is subtracted; to bring neighbours 16 bits apart, a field of codes (at most 16 bits)
// is joined with itself 16 - b bits higher (its top code masked off below, where it would meet the copy's first).  Eight bits go
// through float.
template <int BITS, int N>
__device__ __forceinline__ unsigned apart(unsigned f) {  // f: N codes; a product where the two do not overlap, else an or
  if constexpr (N * BITS <= 16 - BITS)
    return f * (1u + (1u << (16 - BITS)));
  else
    return f | (f << (16 - BITS));
}
template <int BITS, int C0, int N>
__device__ __forceinline__ void decode8(const unsigned (&w)[N], unsigned z, unsigned (&o)[4]) {
  if constexpr (BITS == 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned v = w[(C0 + 2 * i) >> 2] >> (8 * ((C0 + 2 * i) & 3));
      const float a = __uint_as_float(0x4B000000u | (v & 0xffu)) - __uint_as_float(z), b = __uint_as_float(0x4B000000u | ((v >> 8) & 0xffu)) - __uint_as_float(z);
      o[i] = bf2(__floats2bfloat162_rn(a, b));
    }
  } else if constexpr (BITS == 2) {
    // all eight codes at once; those 4 bits up are 8 + c with the exponent of 8
    const unsigned v = C0 % 16 ? w[C0 >> 4] >> 16 : w[C0 >> 4], y = v * 16384u + (v & 0x3fffu);
    const __nv_bfloat162 z4 = __hadd2(bf2(z), __float2bfloat162_rn(120.0f));
    o[0] = bf2(__hadd2(bf2(masked(y, 0x00030003u, 0x43004300u)), bf2(z)));
    o[1] = bf2(__hadd2(bf2(masked(y, 0x00300030u, 0x41004100u)), z4));
    o[2] = bf2(__hadd2(bf2(masked(y >> 8, 0x00030003u, 0x43004300u)), bf2(z)));
    o[3] = bf2(__hadd2(bf2(masked(y >> 8, 0x00300030u, 0x41004100u)), z4));
  } else if constexpr (BITS == 4) {
    const unsigned v = w[C0 >> 3], y0 = v * 4096u + (v & 0xfffu), y1 = (v >> 16) * 4096u + ((v >> 16) & 0xfffu);
    o[0] = bf2(__hadd2(bf2(masked(y0, 0x000f000fu, 0x43004300u)), bf2(z)));
    o[1] = bf2(__hadd2(bf2(masked(y0 >> 8, 0x000f000fu, 0x43004300u)), bf2(z)));
    o[2] = bf2(__hadd2(bf2(masked(y1, 0x000f000fu, 0x43004300u)), bf2(z)));
    o[3] = bf2(__hadd2(bf2(masked(y1 >> 8, 0x000f000fu, 0x43004300u)), bf2(z)));
  } else if constexpr (BITS == 3) {
    constexpr unsigned m = ((1u << BITS) - 1u) * 0x10001u;
    const unsigned y0 = apart<BITS, 4>(field<C0 * BITS, 4 * BITS>(w)), y1 = apart<BITS, 4>(field<(C0 + 4) * BITS, 4 * BITS>(w));
    o[0] = bf2(__hadd2(bf2(masked(y0, m, 0x43004300u)), bf2(z)));
    o[1] = bf2(__hadd2(bf2(masked((y0 >> (2 * BITS)), m, 0x43004300u)), bf2(z)));
    o[2] = bf2(__hadd2(bf2(masked(y1, m, 0x43004300u)), bf2(z)));
    o[3] = bf2(__hadd2(bf2(masked((y1 >> (2 * BITS)), m, 0x43004300u)), bf2(z)));
  } else {
    constexpr unsigned m = ((1u << BITS) - 1u) * 0x10001u;
    const unsigned y0 = apart<BITS, 2>(field<C0 * BITS, 2 * BITS>(w)), y1 = apart<BITS, 2>(field<(C0 + 2) * BITS, 2 * BITS>(w));
    const unsigned y2 = apart<BITS, 2>(field<(C0 + 4) * BITS, 2 * BITS>(w)), y3 = apart<BITS, 2>(field<(C0 + 6) * BITS, 2 * BITS>(w));
    o[0] = bf2(__hadd2(bf2(masked(y0, m, 0x43004300u)), bf2(z)));
    o[1] = bf2(__hadd2(bf2(masked(y1, m, 0x43004300u)), bf2(z)));
    o[2] = bf2(__hadd2(bf2(masked(y2, m, 0x43004300u)), bf2(z)));
    o[3] = bf2(__hadd2(bf2(masked(y3, m, 0x43004300u)), bf2(z)));
  }
}

}  // namespace tb
