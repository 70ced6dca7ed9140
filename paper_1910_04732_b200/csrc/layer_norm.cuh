// Layer norm of token rows, forward and backward, with the residual sum and the dropout in front of it in the same pass.
//   forward : s = R + dropout(X), rounded to the rows' type (that is what S holds and what the blocks behind read, so it is also
//             what is normalised: the result is that of the separate calls);  y = (s - mean) rstd w + b
//   backward: x^ = (s - mean) rstd, a = dy w;  g = rstd (a - mean(a) - x^ mean(a x^)) + dS;  dR = g, dX = dropout'(g);
//             dw = sum_t dy x^, db = sum_t dy
// Sums, means and the deviation are fp32; the variance is the mean of squared differences from the mean (a second look at the row).
#pragma once
#include "dropout.cuh"

namespace flop {
namespace norm {

struct FwdArgs {
  const void* X; int64_t ldx;
  const void* R; int64_t ldr;       // nullable
  void* S; int64_t lds;             // nullable
  void* Y; int64_t ldy;
  const float* w; const float* b;   // nullable: ones, zeros
  float2* stats;                    // nullable: (mean, rstd) of each row
  float eps;
  int64_t T;
  int d, groups, vec, wvec;
  Drop drop;
};

struct BwdArgs {
  const void* dY; int64_t lddy;
  const void* S; int64_t lds;
  const float2* stats;
  const float* w;                   // nullable
  const void* dS; int64_t ldds;     // nullable
  void* dX; int64_t lddx;           // nullable
  void* dR; int64_t lddr;           // nullable
  float* part; int64_t part_ld; int n_part;   // column sums: [n_part][2][part_ld]
  int64_t T;
  int d, groups, vec, wvec;
  Drop drop;
};

// w or b of a group; where the pointer is null, `dflt`
__device__ __forceinline__ void vector8(const float* p, int k, int n, bool vec, float dflt, float (&v)[8]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = dflt;
  } else if (vec && n >= 8) {
    *reinterpret_cast<float4*>(v) = __ldg(reinterpret_cast<const float4*>(p + k));
    *reinterpret_cast<float4*>(v + 4) = __ldg(reinterpret_cast<const float4*>(p + k) + 1);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? __ldg(p + k + j) : 0.f;
  }
}

// What is normalised, rounded to T: s = R + dropout(X).
template <typename T, bool SUM>
__device__ __forceinline__ Raw8<T> summed(const FwdArgs& a, const Raw8<T>& xr, const Raw8<T>& rr, int n, uint64_t ctr) {
  if constexpr (!SUM) return xr;
  float x[8], r[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  unpack8(xr, n, x);
  if (a.R) unpack8(rr, n, r);
  if (a.drop.threshold) {
    const uint4 bits = drop_bits(a.drop, ctr);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = drop_keeps(bits, j, a.drop.threshold) ? fmaf(x[j], a.drop.scale, r[j]) : r[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += r[j];
  }
  return pack8<T>(x);
}

// Sum over the block in a fixed order; every thread gets it.  `scratch` holds a float per warp and is free again at the next sum's barrier.
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (warps == 1) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane == 0) scratch[i * 32 + warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.f;
    for (int w = 0; w < warps; ++w) v[i] += scratch[i * 32 + w];
  }
}

// A block per row that walks the row three times (mean, variance, result): any width.
template <typename T, bool SUM>
__global__ void __launch_bounds__(512)
fwd_walk_kernel(const FwdArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float scratch[32];
  const uint64_t offset = SUM ? drop_offset(a.drop) : 0;
  const int64_t t = blockIdx.x;
  const bool inner = t + 1 < a.T;
  const T* X = (const T*)a.X + t * a.ldx;
  const T* R = SUM && a.R ? (const T*)a.R + t * a.ldr : nullptr;
  T* S = SUM && a.S ? (T*)a.S + t * a.lds : nullptr;
  auto at = [&](int g, bool first, float (&s)[8]) {     // the group's s; S holds it from the first look on (and may have taken X's or R's place)
    const int n = a.d - g * 8;
    Raw8<T> raw;
    if (S && !first) {
      raw = load8((const T*)S + g * 8, n, a.vec, inner);
    } else {
      raw = load8(X + g * 8, n, a.vec, inner);
      Raw8<T> rr = raw;
      if (R) rr = load8(R + g * 8, n, a.vec, inner);
      raw = summed<T, SUM>(a, raw, rr, n, offset + (uint64_t)t * a.groups + g);
      if (S) store8(S + g * 8, raw, n, a.vec);
    }
    unpack8(raw, n, s);
    return n;
  };
  float sum[1] = {0.f}, s[8];
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    at(g, true, s);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[0] += s[j];
  }
  block_sum(sum, scratch);
  const float mean = sum[0] / (float)a.d;
  sum[0] = 0.f;
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    const int n = at(g, false, s);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[0] += j < n ? (s[j] - mean) * (s[j] - mean) : 0.f;
  }
  block_sum(sum, scratch);
  const float rstd = rsqrtf(sum[0] / (float)a.d + a.eps);
  if (a.stats && threadIdx.x == 0) a.stats[t] = make_float2(mean, rstd);
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    const int n = at(g, false, s);
    float w[8], b[8];
    vector8(a.w, g * 8, n, a.wvec, 1.f, w);
    vector8(a.b, g * 8, n, a.wvec, 0.f, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = fmaf((s[j] - mean) * rstd, w[j], b[j]);
    store8((T*)a.Y + t * a.ldy + g * 8, pack8<T>(s), n, a.vec);
  }
}

// dX and dR of a row, walked twice: any width.
template <typename T>
__global__ void __launch_bounds__(512)
bwd_walk_kernel(const BwdArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float scratch[64];
  const uint64_t offset = drop_offset(a.drop);
  const int64_t t = blockIdx.x;
  const bool inner = t + 1 < a.T;
  const T* dY = (const T*)a.dY + t * a.lddy;
  const T* S = (const T*)a.S + t * a.lds;
  const float2 st = a.stats[t];
  float x[8], dy[8], w[8];
  auto at = [&](int g) {           // x: x^, dy: a = dy w
    const int n = a.d - g * 8;
    const Raw8<T> sr = load8(S + g * 8, n, a.vec, inner), yr = load8(dY + g * 8, n, a.vec, inner);
    vector8(a.w, g * 8, n, a.wvec, 1.f, w);
    unpack8(sr, n, x);
    unpack8(yr, n, dy);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = (x[j] - st.x) * st.y;
      dy[j] *= w[j];
    }
    return n;
  };
  float c[2] = {0.f, 0.f};
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    const int n = at(g);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) { c[0] += dy[j]; c[1] = fmaf(dy[j], x[j], c[1]); }
  }
  block_sum(c, scratch);
  const float c1 = c[0] / (float)a.d, c2 = c[1] / (float)a.d;
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    const int n = at(g);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = st.y * (dy[j] - c1 - x[j] * c2);
    if (a.dS) {
      unpack8(load8((const T*)a.dS + t * a.ldds + g * 8, n, a.vec, inner), n, dy);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] += dy[j];
    }
    if (a.dR) store8((T*)a.dR + t * a.lddr + g * 8, pack8<T>(x), n, a.vec);
    if (a.dX) {
      if (a.drop.threshold) {
        const uint4 bits = drop_bits(a.drop, offset + (uint64_t)t * a.groups + g);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = drop_keeps(bits, j, a.drop.threshold) ? x[j] * a.drop.scale : 0.f;
      }
      store8((T*)a.dX + t * a.lddx + g * 8, pack8<T>(x), n, a.vec);
    }
  }
}

// Column sums of dy x^ and dy over a run of rows: 32 groups across, eight rows at a time; the eight are added in order.
template <typename T>
__global__ void __launch_bounds__(256)
bwd_columns_kernel(const BwdArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float red[8][32][9];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = blockIdx.x * 32 + lane, n = a.d - g * 8;
  const int64_t per = (a.T + gridDim.y - 1) / gridDim.y, t0 = blockIdx.y * per, t1 = min(a.T, t0 + per);
  float dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, db[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int64_t t = t0 + warp; t < t1; t += 8) {
    const bool inner = t + 1 < a.T;
    const Raw8<T> sr = load8((const T*)a.S + t * a.lds + g * 8, n, a.vec, inner), yr = load8((const T*)a.dY + t * a.lddy + g * 8, n, a.vec, inner);
    const float2 st = a.stats[t];
    float x[8], dy[8];
    unpack8(sr, n, x);
    unpack8(yr, n, dy);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw[j] = fmaf(dy[j], (x[j] - st.x) * st.y, dw[j]);
      db[j] += dy[j];
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) red[warp][lane][j] = h ? db[j] : dw[j];
    __syncthreads();
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k < a.d) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) s += red[r][threadIdx.x >> 3][threadIdx.x & 7];
      a.part[((int64_t)blockIdx.y * 2 + h) * a.part_ld + k] = s;
    }
  }
}

// dweight and dbias (=|+=) the partial sums of a column: 32 columns a block, a warp adds a run of the partials, the runs are added in order.
__global__ void __launch_bounds__(256)
bwd_finish_kernel(const float* __restrict__ part, int64_t part_ld, int n_part, int d, float* dweight, float* dbias, int accumulate) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.x * 32 + lane;
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  const int per = (n_part + 7) / 8, p1 = min(n_part, (warp + 1) * per);
  float s = 0.f;
  if (k < d) {
#pragma unroll 8
    for (int p = warp * per; p < p1; ++p) s += part[((int64_t)p * 2 + blockIdx.y) * part_ld + k];
  }
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && k < d) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w][lane];
    out[k] = accumulate ? out[k] + s : s;
  }
}

}  // namespace norm
}  // namespace flop
