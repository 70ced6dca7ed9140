// The library's counter-based generator.
#pragma once
#include <stdint.h>

namespace flop {

__device__ __forceinline__ uint4 philox4x32_10(uint4 c, uint2 k) {
  // Philox-4x32, ten rounds (Salmon et al., SC'11): two 32x32->64 multiplies
  // per round, xor with the key and the neighbouring words, Weyl key schedule.
  constexpr uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint32_t hi0 = __umulhi(M0, c.x), lo0 = M0 * c.x;
    const uint32_t hi1 = __umulhi(M1, c.z), lo1 = M1 * c.z;
    c = make_uint4(hi1 ^ c.y ^ k.x, lo1, hi0 ^ c.w ^ k.y, lo0);
    k.x += W0;
    k.y += W1;
  }
  return c;
}

}  // namespace flop
