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

// fp32 quotients are off by less than 127 * 3 * 2^-24 = 2.3e-5.
constexpr float kBorder = 1e-4f;

__device__ __forceinline__ int round_exact(double x, double amax) { return (int)rint(127.0 * x / amax); }
// `inv` = 127 / amax in fp32 (infinite for the smallest amax, then every value takes the fp64 path)
__device__ __forceinline__ int quantize(float x, float inv, float amax) {
  const float y = x * inv, n = rintf(y);
  if (!(fabsf(y - n) < 0.5f - kBorder)) return round_exact((double)x, (double)amax);
  return (int)n;
}

constexpr int kRowThreads = 128;

__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < (int)blockDim.x / 32; ++w) v = fmaxf(v, red[w]);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
quantize_rows_kernel(const T* __restrict__ X, int64_t ldx, int cols, int8_t* __restrict__ Xq, int64_t ldq, float* __restrict__ scale) {
  __shared__ float red[32];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = blockIdx.x;
  X += row * ldx; Xq += row * ldq;
  float amax = 0.f;
  bool bad = false;
  for (int c = threadIdx.x; c < cols; c += kRowThreads) {
    const float x = fabsf(to_f32(X[c]));
    bad |= !(x < INFINITY);
    amax = fmaxf(amax, x);
  }
  bad = __syncthreads_or(bad);
  amax = block_max(amax, red);
  const bool zero = bad || amax == 0.f;
  const float inv = 127.f / amax;
  for (int c = threadIdx.x; c < cols; c += kRowThreads) Xq[c] = zero ? 0 : (int8_t)quantize(to_f32(X[c]), inv, amax);
  if (threadIdx.x == 0) scale[row] = bad ? NAN : amax / 127.f;
}

// H in 32-bit sums times the scale of its column, requantised per row: h = acc * col_scale, exact in fp64 as long as the
// sum has 29 bits, hq = 127 h / max |h| rounded, h_scale = row_scale * max |h| / 127.
__global__ void __launch_bounds__(kRowThreads)
requantize_rows_kernel(const int* __restrict__ acc, int64_t lda, int cols, const float* __restrict__ col_scale, const float* __restrict__ row_scale,
                       int8_t* __restrict__ Hq, int64_t ldq, float* __restrict__ h_scale) {
  __shared__ double red[32];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = blockIdx.x;
  acc += row * lda; Hq += row * ldq;
  double amax = 0.0;
  bool bad = false;
  for (int c = threadIdx.x; c < cols; c += kRowThreads) {
    const double h = fabs((double)acc[c] * (double)col_scale[c]);
    bad |= !(h < INFINITY);
    amax = fmax(amax, h);
  }
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
  __syncthreads();
  amax = red[0];
  for (int w = 1; w < kRowThreads / 32; ++w) amax = fmax(amax, red[w]);
  const bool zero = bad || amax == 0.0;
  for (int c = threadIdx.x; c < cols; c += kRowThreads) Hq[c] = zero ? 0 : (int8_t)round_exact((double)acc[c] * (double)col_scale[c], amax);
  if (threadIdx.x == 0) h_scale[row] = bad ? NAN : (float)((double)row_scale[row] * (amax / 127.0));
}

}  // namespace i8
}  // namespace flop
