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

struct DropoutArgs {
  const void* X; int64_t ldx;
  const void* R; int64_t ldr;
  void* Y; int64_t ldy;
  int64_t T, total;                 // rows, groups of all rows
  int d, groups;                    // columns, groups of a row
  int64_t step_rows; int step_groups;   // what the grid's stride is in rows and groups
  int vec;
  Drop drop;
};

template <typename T, bool RES>
__global__ void __launch_bounds__(256)
dropout_kernel(const DropoutArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const uint64_t offset = drop_offset(a.drop);
  int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, t = i / a.groups;
  int g = (int)(i - t * a.groups);
  for (; i < a.total; i += (int64_t)gridDim.x * blockDim.x) {
    const int n = a.d - g * 8;
    const bool inner = t + 1 < a.T;
    const Raw8<T> xr = load8((const T*)a.X + t * a.ldx + g * 8, n, a.vec, inner);
    Raw8<T> rr;
    if (RES) rr = load8((const T*)a.R + t * a.ldr + g * 8, n, a.vec, inner);
    const uint4 bits = drop_bits(a.drop, offset + (uint64_t)i);
    float x[8], r[8];
    unpack8(xr, n, x);
    if (RES) unpack8(rr, n, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool keep = drop_keeps(bits, j, a.drop.threshold);
      if (RES) x[j] = keep ? fmaf(x[j], a.drop.scale, r[j]) : r[j];
      else x[j] = keep ? x[j] * a.drop.scale : 0.f;
    }
    store8((T*)a.Y + t * a.ldy + g * 8, pack8<T>(x), n, a.vec);
    t += a.step_rows;
    g += a.step_groups;
    if (g >= a.groups) { g -= a.groups; ++t; }
  }
}

}  // namespace flop
