// 8-bit integers with a scale per row: the factors of a pruned matrix (a scale per output channel) and the tokens they are
// multiplied with (a scale per token).
//     scale_t = max_c |x_tc| / 127,    q_tc = 127 x_tc / max_c |x_tc|  rounded half to even
// The rounding is decided as in exact arithmetic: in fp32 where the quotient is further than its error from a border, else in fp64,
// which holds 127 x exactly and whose quotient lies on the border only where the exact one does.  So the integers are the
// same whichever kernel makes them.  A row of zeros has scale 0; a row with an infinity or a NaN has scale NaN and zeros, so that what is
// computed from it is NaN.
#pragma once
#include "common.cuh"

namespace flop {
namespace i8 {

// x * (127 / amax) in fp32 is off by one rounding of the factor and one of the product, 127 * 2^-23 = 1.5e-5 at most (the fused residual
// has no product rounding: half of it); with x itself a product of two rounded factors and amax rounded, by 127 * 2^-24 * 5 = 3.8e-5.
constexpr float kBorder = 2e-5f, kBorderSums = 5e-5f;
constexpr float kToInt = 12582912.f;              // 1.5 * 2^23: adding it rounds to an integer, which is then the sum's low bits

// 127 x / amax for a quotient within kBorder of lower + 1/2: 254 x against (2 lower + 1) amax, both as a product and its rounding error, so
// that the comparison is exact; half goes to even.
template <typename F>
__device__ __forceinline__ int round_border(F x, F amax, int lower) {
  const F odd = (F)(2 * lower + 1), p = (F)254 * x, q = odd * amax;
  const F d = (p - q) + (fma((F)254, x, -p) - fma(odd, amax, -q));
  return lower + (d > (F)0 || (d == (F)0 && (lower & 1)));
}

__device__ __forceinline__ int round_exact(double x, double amax) { return (int)rint(127.0 * x / amax); }
// Eight values' low bytes.
__device__ __forceinline__ uint2 bytes8(const uint32_t (&b)[8]) {
  return make_uint2(__byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410));
}
}  // namespace i8
}  // namespace flop
