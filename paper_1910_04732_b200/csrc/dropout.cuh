// Dropout whose mask is a function of (seed, counter) and is never stored: Y = R + keep X s, and backwards dX = keep dY s.
//
// Group g of row t (columns 8g .. 8g+7) takes ONE Philox block, counter offset + t ceil(d / 8) + g, third counter word 1 (the gates'
// sampler has 0 there: the same seed gives other numbers).  Its 128 bits are eight 16-bit values h, column j the j-th; the column is
// kept where h >= threshold, threshold = p in units of 2^-16 (nearest), and s = 65536 / (65536 - threshold), so the expectation of
// what is kept is exact for the probability that is drawn.  16 bits a value: ten rounds are about 60 integer instructions, and with
// 32 bits a value (four to a block) they would take as long as the memory traffic of bf16 rows.
#pragma once
#include "philox.cuh"
#include "rows8.cuh"

namespace flop {

struct Drop {
  uint2 key;
  uint64_t offset;
  const uint64_t* offset_dev;       // nullable: added to offset, so that a captured launch can draw anew
  uint32_t threshold;               // 0: nothing is dropped
  float scale;
};

__device__ __forceinline__ uint64_t drop_offset(const Drop& d) { return d.offset + (d.offset_dev ? *d.offset_dev : 0ull); }
__device__ __forceinline__ uint4 drop_bits(const Drop& d, uint64_t ctr) {
  return philox4x32_10(make_uint4((uint32_t)ctr, (uint32_t)(ctr >> 32), 1u, 0u), d.key);
}
__device__ __forceinline__ bool drop_keeps(const uint4& x, int j, uint32_t threshold) {
  const uint32_t w = j < 2 ? x.x : j < 4 ? x.y : j < 6 ? x.z : x.w;
  return (j & 1 ? w >> 16 : w & 0xFFFFu) >= threshold;
}
// The bits of a thread's NU units, 16 for each column; group(i): the counter of unit i's group.  A unit of fp32 is half a group: the even thread of a pair has the first
// half of both threads' groups, the odd one the second; each draws every other group and they exchange halves.  All lanes of a warp come here
// together.
template <typename T, int NU, typename F>
__device__ __forceinline__ void drop_units(const Drop& d, bool odd, F&& group, uint32_t (&bits)[NU][kPairs<T>]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const uint4 x = drop_bits(d, group(i));
      bits[i][0] = x.x; bits[i][1] = x.y; bits[i][2] = x.z; bits[i][3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NU; i += 2) {
      const uint64_t even_group = group(i), odd_group = group(i + 1 < NU ? i + 1 : i);
      const uint4 x = drop_bits(d, odd ? odd_group : even_group);
      const uint32_t keep[2] = {odd ? x.z : x.x, odd ? x.w : x.y};
      if (i + 1 < NU) {
        const uint32_t got[2] = {__shfl_xor_sync(0xffffffffu, odd ? x.x : x.z, 1), __shfl_xor_sync(0xffffffffu, odd ? x.y : x.w, 1)};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          bits[i][j] = odd ? got[j] : keep[j];
          bits[i + 1 < NU ? i + 1 : i][j] = odd ? keep[j] : got[j];
        }
      } else {
        bits[i][0] = keep[0];
        bits[i][1] = keep[1];
      }
    }
  }
}
__device__ __forceinline__ uint64_t select_pair(uint32_t bits, uint32_t threshold, uint64_t kept, uint64_t dropped) {
  const float2 k = unpack2(kept), d = unpack2(dropped);
  const uint32_t above = threshold << 16;                // what is below the half compared does not matter
  return pack2((bits << 16) >= above ? k.x : d.x, bits >= above ? k.y : d.y);
}

}  // namespace flop
