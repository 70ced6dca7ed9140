// Layer norm of token rows, forward and backward, with the residual sum and the dropout in front of it in the same pass.
//   forward : s = R + dropout(X), the product and the sum in fp32, rounded to the rows' type (that is what S holds and what the blocks behind read, so it is also
//             what is normalised: the result is that of the separate calls);  y = (s - mean) rstd w + b
//   backward: x^ = (s - mean) rstd, a = dy w;  g = rstd (a - mean(a) - x^ mean(a x^)) + dS;  dR = g, dX = dropout'(g);
//             dw = sum_t dy x^, db = sum_t dy
// Sums, means and the deviation are fp32; the variance is the mean of squared differences from the mean (a second look at the row).
//
// A row of equal values has differences of exactly 0, so that its result is the bias: its mean has to be the value to the last bit, whatever the width.
//   bf16 : sums of up to 16384 equal values take 22 bits and are exact, and divided() gives a quotient that is representable as it is
//   fp32 : sums round, and the mean is a few steps of the value off.  Where the deviation is below 2^-12 of the mean, so that this could be seen, the differences are added up and what
//          they are off by on average is taken from them and given to the mean: of equal values they are k steps each, k below 64 (a sum of 16384 passes through at most 45 additions), and d k
//          steps are exact.  Other rows pay a comparison (8192 x 1024 11.2 us; every row corrected 13.9, summed in fp64 13.4).
//   walked rows are summed in fp64: 2^23 equal values take 47 bits
#pragma once
#include <type_traits>

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
  double inv_d;                     // for sums in fp64
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
  float* part; int64_t part_ld; int n_part;   // column sums: [n_part][2][part_ld] (null: not wanted)
  float* dweight; float* dbias; int accumulate;
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
    for (int j = 0; j < 8; ++j) x[j] = __fadd_rn(drop_keeps(bits, j, a.drop.threshold) ? __fmul_rn(x[j], a.drop.scale) : 0.f, r[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += r[j];
  }
  return pack8<T>(x);
}

// Sum over the block in a fixed order; every thread gets it.  `scratch` holds a value per warp and is free again at the next sum's barrier.
template <typename V, int N>
__device__ __forceinline__ void block_sum(V (&v)[N], V* scratch) {
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
    v[i] = 0;
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
  __shared__ double total_scratch[32];
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
  double total[1] = {0.};
  float sum[1] = {0.f}, s[8];
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    at(g, true, s);
    if constexpr (sizeof(T) == 2) {                        // eight equal values take 11 bits; two of fp32 as many as one
      total[0] += (double)(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    } else {
#pragma unroll
      for (int j = 0; j < 8; j += 2) total[0] += (double)(s[j] + s[j + 1]);
    }
  }
  block_sum(total, total_scratch);
  const float mean = (float)(total[0] * a.inv_d);
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

// ---------------------------------------------------------------- rows held in registers, copied ahead
// A row is shared by LANES threads, NG units of 16 bytes each (8 columns of bf16, 4 of fp32; a unit is LANES units behind the thread's one before, so
// that a warp's accesses are contiguous), always the same columns: weights, and in the backward pass the column sums, stay in
// registers from row to row.  A block works on RB rows of each set of LANES threads at once and walks every gridDim.x-th batch;
// every thread copies its own units of the next STAGES batches to shared memory asynchronously and reads them back itself, so nothing has to be
// waited for but the thread's own copies, and the memory system always has work in flight: under load an access takes 1.5 to 2 us, and a
// kernel that loads, computes and stores a row at a time has a quarter of the bytes in flight that this needs.
// All units but the last of a thread are whole and present (the host picks LANES and NG so), which leaves one to be looked at.
// The thread's units of a row (`from`: its first), `last` columns in the last one (<= 0: none), into its slots, THREADS apart.  No such row (on is false): zeros.
// EACH: any of its units may end early or be absent.
template <typename T, int LANES, int NG, int THREADS, bool EACH = false>
__device__ __forceinline__ void copy_units(uint4* to, const T* from, int last, bool on, bool vec) {
#pragma unroll
  for (int i = 0; i < NG; ++i)
    copy_unit(to + i * THREADS, from + i * LANES * kUnit<T>, !on ? 0 : EACH ? last + (NG - 1 - i) * LANES * kUnit<T> : i < NG - 1 ? kUnit<T> : last, vec);
}
// Pairs of a vector's columns; absent ones 0.
template <typename T>
__device__ __forceinline__ void vector_unit(const float* p, int k, int n, bool vec, float dflt, uint64_t (&v)[kPairs<T>]) {
  float f[kUnit<T>];
#pragma unroll
  for (int j = 0; j < kUnit<T>; j += 4) {
    if (p && vec && n >= j + 4) {
      *reinterpret_cast<float4*>(f + j) = __ldg(reinterpret_cast<const float4*>(p + k + j));
    } else {
#pragma unroll
      for (int i = j; i < j + 4; ++i) f[i] = i < n ? (p ? __ldg(p + k + i) : dflt) : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < kPairs<T>; ++j) v[j] = pack2(f[2 * j], f[2 * j + 1]);
}

// Sums over the LANES threads that share a row, in a fixed order; every one gets them.  Rows of several warps have a barrier each; `scratch` (one
// of two, in turn) is free again once the sum after the next begins.
template <int LANES, int THREADS, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*scratch)[32]) {
#pragma unroll
  for (int o = (LANES < 32 ? LANES : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (LANES > 32) {
    const int warp = threadIdx.x >> 5, first = warp / (LANES / 32) * (LANES / 32);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) scratch[i][warp] = v[i];
    }
    if constexpr (LANES == THREADS) __syncthreads();     // a barrier named at run time would take all of a block's barriers, and so keep blocks from the SM
    else asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.x / LANES + 1), "n"(LANES) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < LANES / 32; ++w) v[i] += scratch[i][first + w];
    }
  }
}
__device__ __forceinline__ float both(uint64_t v) {
  const float2 u = unpack2(v);
  return u.x + u.y;
}
// sum / d: what the product with 1 / d (inv_d, rounded) leaves over is divided too.
__device__ __forceinline__ float divided(float sum, float d, float inv_d) {
  const float q = sum * inv_d;
  return fmaf(fmaf(-q, d, sum), inv_d, q);
}

// What the forward kernel does with a row: WHOLE is the norm of X, SUMMED that of S = R + dropout(X); ADDED and DROPPED stop at S, with and without R: dropout by itself, which
// has no use for whole rows, so that a row may be cut into segments of LANES * NG units (blockIdx.y).
enum { WHOLE, SUMMED, ADDED, DROPPED };
template <int MODE> constexpr int kTensors = MODE == SUMMED || MODE == ADDED ? 2 : 1;
template <int MODE> constexpr bool kNorm = MODE == WHOLE || MODE == SUMMED;
template <typename T, int MODE, int LANES, int NG, int RB, int STAGES, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS)
fwd_kernel(const FwdArgs a) {
  constexpr bool SUM = MODE != WHOLE, NORM = kNorm<MODE>, RES = kTensors<MODE> == 2;
  constexpr int ROWS = THREADS / LANES, E = kUnit<T>, H = kPairs<T>, ROW = NG * THREADS, SIZE = kTensors<MODE> * RB * ROW;
  extern __shared__ uint4 ring[];                        // [STAGES][X and R][RB][NG][THREADS]
  __shared__ float scratch[sizeof(T) == 4 ? 4 : 2][RB][32];
  const int l = threadIdx.x % LANES + (NORM ? 0 : blockIdx.y * LANES * NG), r = threadIdx.x / LANES;
  const int last = a.d - (l + (NG - 1) * LANES) * E;     // columns of the last unit
  const int batches = (int)((a.T + ROWS * RB - 1) / (ROWS * RB));
  const float d = (float)a.d, inv_d = 1.f / d;
  pdl_wait();
  pdl_launch_dependents();
  const uint64_t offset = SUM ? drop_offset(a.drop) : 0, scale = SUM ? pack2(a.drop.scale, a.drop.scale) : 0;
  auto fetch = [&](int batch, int stage) {
    uint4* to = ring + stage * SIZE + threadIdx.x;
#pragma unroll
    for (int q = 0; q < RB; ++q) {
      const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
      copy_units<T, LANES, NG, THREADS, !NORM>(to + q * ROW, (const T*)a.X + t * a.ldx + l * E, last, t < a.T, a.vec);
      if (RES && a.R) copy_units<T, LANES, NG, THREADS, !NORM>(to + (RB + q) * ROW, (const T*)a.R + t * a.ldr + l * E, last, t < a.T, a.vec);
    }
  };
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
    const int batch = blockIdx.x + st * gridDim.x;
    if (batch < batches) fetch(batch, st);
    copies_commit();
  }
  uint64_t w[NORM ? NG : 1][H], b[NORM ? NG : 1][H];
  if constexpr (NORM) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int k = (l + i * LANES) * E;
      vector_unit<T>(a.w, k, a.d - k, a.wvec, 1.f, w[i]);
      vector_unit<T>(a.b, k, a.d - k, a.wvec, 0.f, b[i]);
    }
  }
  auto rows = [&](auto known) {                          // dropout: 0 no, 1 yes, 2 as the arguments say
    constexpr int KNOWN = decltype(known)::value;
    const bool drops = KNOWN == 2 ? a.drop.threshold != 0 : KNOWN == 1;
    int stage = 0;
    for (int batch = blockIdx.x; batch < batches; batch += gridDim.x) {
      copies_wait<STAGES - 1>();
      const uint4* at = ring + stage * SIZE + threadIdx.x;
      uint64_t s[NORM ? RB : 1][NORM ? NG : 1][H];
      float sum[RB];
#pragma unroll
      for (int q = 0; q < RB; ++q) {
        const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
        uint64_t total = 0;
        uint32_t bits[NG][H];
        if (SUM && (!RES || drops)) drop_units<T, NG>(a.drop, l & 1, [&](int i) { return offset + (uint64_t)t * a.groups + (uint32_t)((l + i * LANES) / (8 / E)); }, bits);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          uint64_t(&v)[H] = s[NORM ? q : 0][NORM ? i : 0];
          unpack_unit<T>(at[q * ROW + i * THREADS], v);
          if constexpr (SUM) {
            uint64_t res[H];
            if (RES && a.R) {
              unpack_unit<T>(at[(RB + q) * ROW + i * THREADS], res);
            } else {
#pragma unroll
              for (int j = 0; j < H; ++j) res[j] = 0;
            }
#pragma unroll
            for (int j = 0; j < H; ++j) {
              if (!RES || drops) v[j] = select_pair(bits[i][j], a.drop.threshold, mul2(v[j], scale), 0);
              if (RES) v[j] = add2(v[j], res[j]);
            }
            const uint4 rounded = pack_unit<T>(v);
            const int n = !NORM ? last + (NG - 1 - i) * LANES * E : i < NG - 1 ? E : last;
            if (a.S && t < a.T && n > 0) store_unit((T*)a.S + t * a.lds + (l + i * LANES) * E, rounded, n, a.vec);
            if (NORM) unpack_unit<T>(rounded, v);
          }
          if constexpr (NORM) {
#pragma unroll
            for (int j = 0; j < H; ++j) total = add2(total, v[j]);
          }
        }
        sum[q] = both(total);
      }
      const int ahead = batch + STAGES * gridDim.x;
      if (ahead < batches) fetch(ahead, stage);
      copies_commit();
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      if constexpr (NORM) {
        row_sum<LANES, THREADS>(sum, scratch[0]);
        float mean[RB];
        auto less = [&](int q, float by) {                   // the row's values less `by`; the sum of this thread's squares
          const uint64_t minus = pack2(-by, -by);
          uint64_t total = 0;
#pragma unroll
          for (int i = 0; i < NG; ++i) {
#pragma unroll
            for (int j = 0; j < H; ++j) s[q][i][j] = add2(s[q][i][j], minus);
            if (i == NG - 1 && last < E) {                   // what lies behind the row's end is no difference
#pragma unroll
              for (int j = 0; j < H; ++j) {
                const float2 u = unpack2(s[q][i][j]);
                s[q][i][j] = pack2(2 * j < last ? u.x : 0.f, 2 * j + 1 < last ? u.y : 0.f);
              }
            }
#pragma unroll
            for (int j = 0; j < H; ++j) total = fma2(s[q][i][j], s[q][i][j], total);
          }
          return both(total);
        };
#pragma unroll
        for (int q = 0; q < RB; ++q) {
          mean[q] = divided(sum[q], d, inv_d);
          sum[q] = less(q, mean[q]);
        }
        row_sum<LANES, THREADS>(sum, scratch[1]);
        if constexpr (sizeof(T) == 4) {                      // rows whose values are nearly equal; all threads of a row agree on it
          auto close = [&](int q) { return sum[q] <= mean[q] * mean[q] * (d * 0x1p-24f) && mean[q] != 0.f; };     // also where squares are too small to be held
          bool any = false;
#pragma unroll
          for (int q = 0; q < RB; ++q) any |= close(q);
          if (LANES < 32) any = __any_sync(0xffffffffu, any);
          if (any) {
            float off[RB], square[RB];
#pragma unroll
            for (int q = 0; q < RB; ++q) {
              uint64_t total = 0;
#pragma unroll
              for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int j = 0; j < H; ++j) total = add2(total, s[q][i][j]);
              off[q] = both(total);
            }
            row_sum<LANES, THREADS>(off, scratch[2]);
#pragma unroll
            for (int q = 0; q < RB; ++q) {
              off[q] = close(q) ? divided(off[q], d, inv_d) : 0.f;       // a row's result does not depend on its neighbours
              mean[q] += off[q];
              square[q] = less(q, off[q]);
            }
            row_sum<LANES, THREADS>(square, scratch[3]);
#pragma unroll
            for (int q = 0; q < RB; ++q) sum[q] = square[q];
          }
        }
#pragma unroll
        for (int q = 0; q < RB; ++q) {
          const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
          if (t >= a.T) break;
          const float rstd = rsqrtf(fmaf(sum[q], inv_d, a.eps));
          if (a.stats && l == 0) a.stats[t] = make_float2(mean[q], rstd);
          const uint64_t by = pack2(rstd, rstd);
          T* Y = (T*)a.Y + t * a.ldy + l * E;
#pragma unroll
          for (int i = 0; i < NG; ++i) {
            const int n = i < NG - 1 ? E : last;
            if (n > 0) {
#pragma unroll
              for (int j = 0; j < H; ++j) s[q][i][j] = fma2(mul2(s[q][i][j], by), w[i][j], b[i][j]);
              store_unit(Y + i * LANES * E, pack_unit<T>(s[q][i]), n, a.vec);
            }
          }
        }
      }
    }
  };
  // Twice for sums of fp32: a condition in the loop keeps the generator's rounds from being spread among the row's other work (9000 x 410 16.6 us, 13.5 now).
  if constexpr (sizeof(T) == 4 && MODE == SUMMED) {
    if (a.drop.threshold) rows(std::integral_constant<int, 1>{});
    else rows(std::integral_constant<int, 0>{});
  } else {
    rows(std::integral_constant<int, 2>{});
  }
}

// Backward: the same, and with the rows the running column sums.  x^ and a are formed twice, from the ring, before and after the row's sums are known: kept in
// registers beside the column sums they cost 40 registers and a quarter of the warps (16384 x 2048 bf16: 45 against 41 us).  The block's sums go
// to its place in the workspace or, where it is the only block, to dweight and dbias.
template <typename T, int LANES, int NG, int RB, int STAGES, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS)
bwd_kernel(const BwdArgs a) {
  constexpr int ROWS = THREADS / LANES, E = kUnit<T>, H = kPairs<T>, ROW = NG * THREADS;
  extern __shared__ uint4 ring[];                        // [STAGES][S, dY and, where there is one, dS][RB][NG][THREADS]
  __shared__ float scratch[2][2 * RB][32];
  const int size = (a.dS ? 3 : 2) * RB * ROW;
  const int l = threadIdx.x % LANES, r = threadIdx.x / LANES;
  const int last = a.d - (l + (NG - 1) * LANES) * E;
  const int batches = (int)((a.T + ROWS * RB - 1) / (ROWS * RB));
  const float inv_d = 1.f / (float)a.d;
  pdl_wait();
  pdl_launch_dependents();
  const uint64_t offset = drop_offset(a.drop), scale = pack2(a.drop.scale, a.drop.scale);
  auto fetch = [&](int batch, int stage) {
    uint4* to = ring + stage * size + threadIdx.x;
#pragma unroll
    for (int q = 0; q < RB; ++q) {
      const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
      copy_units<T, LANES, NG, THREADS>(to + q * ROW, (const T*)a.S + t * a.lds + l * E, last, t < a.T, a.vec);
      copy_units<T, LANES, NG, THREADS>(to + (RB + q) * ROW, (const T*)a.dY + t * a.lddy + l * E, last, t < a.T, a.vec);
      if (a.dS) copy_units<T, LANES, NG, THREADS>(to + (2 * RB + q) * ROW, (const T*)a.dS + t * a.ldds + l * E, last, t < a.T, a.vec);
    }
  };
  float2 next[RB];                                       // (mean, rstd) of the next batch's rows
  auto fetch_stats = [&](int batch) {
#pragma unroll
    for (int q = 0; q < RB; ++q) {
      const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
      next[q] = t < a.T ? a.stats[t] : make_float2(0.f, 0.f);
    }
  };
  fetch_stats(blockIdx.x);
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
    const int batch = blockIdx.x + st * gridDim.x;
    if (batch < batches) fetch(batch, st);
    copies_commit();
  }
  uint64_t w[NG][H], dw[NG][H], db[NG][H];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int k = (l + i * LANES) * E;
    vector_unit<T>(a.w, k, a.d - k, a.wvec, 1.f, w[i]);
#pragma unroll
    for (int j = 0; j < H; ++j) dw[i][j] = db[i][j] = 0;
  }
  int stage = 0, turn = 0;
  for (int batch = blockIdx.x; batch < batches; batch += gridDim.x) {
    float2 st[RB];
#pragma unroll
    for (int q = 0; q < RB; ++q) st[q] = next[q];
    if (batch + (int)gridDim.x < batches) fetch_stats(batch + gridDim.x);
    copies_wait<STAGES - 1>();
    const uint4* at = ring + stage * size + threadIdx.x;
    uint64_t xv[H], yv[H];                               // x^; dy, then a = dy w
    auto load = [&](int q, int i) {
      const uint64_t minus = pack2(-st[q].x, -st[q].x), by = pack2(st[q].y, st[q].y);
      unpack_unit<T>(at[q * ROW + i * THREADS], xv);
      unpack_unit<T>(at[(RB + q) * ROW + i * THREADS], yv);                               // 0 behind the row's end, and so is what is added up
#pragma unroll
      for (int j = 0; j < H; ++j) xv[j] = mul2(add2(xv[j], minus), by);
    };
    float c[2 * RB];
#pragma unroll
    for (int q = 0; q < RB; ++q) {
      uint64_t c0 = 0, c1 = 0;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        load(q, i);
#pragma unroll
        for (int j = 0; j < H; ++j) {
          dw[i][j] = fma2(yv[j], xv[j], dw[i][j]);
          db[i][j] = add2(db[i][j], yv[j]);
          yv[j] = mul2(yv[j], w[i][j]);
          c0 = add2(c0, yv[j]);
          c1 = fma2(yv[j], xv[j], c1);
        }
      }
      c[2 * q] = both(c0);
      c[2 * q + 1] = both(c1);
    }
    if (a.dX || a.dR) {
      row_sum<LANES, THREADS>(c, scratch[turn]);
      turn ^= 1;
#pragma unroll
      for (int q = 0; q < RB; ++q) {
        const int64_t t = ((int64_t)batch * RB + q) * ROWS + r;
        const bool on = t < a.T;
        const float c1 = -c[2 * q] * inv_d, c2 = -c[2 * q + 1] * inv_d;
        const uint64_t m1 = pack2(c1, c1), m2 = pack2(c2, c2), by = pack2(st[q].y, st[q].y);
        uint32_t bits[NG][H];
        if (a.dX && a.drop.threshold) drop_units<T, NG>(a.drop, l & 1, [&](int i) { return offset + (uint64_t)t * a.groups + (uint32_t)((l + i * LANES) / (8 / E)); }, bits);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int k = (l + i * LANES) * E, n = i < NG - 1 ? E : last;
          load(q, i);
#pragma unroll
          for (int j = 0; j < H; ++j) yv[j] = mul2(fma2(xv[j], m2, fma2(yv[j], w[i][j], m1)), by);
          if (a.dS) {
            uint64_t e[H];
            unpack_unit<T>(at[(2 * RB + q) * ROW + i * THREADS], e);
#pragma unroll
            for (int j = 0; j < H; ++j) yv[j] = add2(yv[j], e[j]);
          }
          if (on && n > 0) {
            if (a.dR) store_unit((T*)a.dR + t * a.lddr + k, pack_unit<T>(yv), n, a.vec);
            if (a.dX) {
              if (a.drop.threshold) {
#pragma unroll
                for (int j = 0; j < H; ++j) yv[j] = select_pair(bits[i][j], a.drop.threshold, mul2(yv[j], scale), 0);
              }
              store_unit((T*)a.dX + t * a.lddx + k, pack_unit<T>(yv), n, a.vec);
            }
          }
        }
      }
    }
    const int ahead = batch + STAGES * gridDim.x;
    if (ahead < batches) fetch(ahead, stage);
    copies_commit();
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  if (!a.part) return;
  const bool only = gridDim.x == 1;
  float* out[2] = {only ? a.dweight : a.part + (int64_t)blockIdx.x * 2 * a.part_ld, only ? a.dbias : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.part_ld};
  auto put = [&](int h, int k, float v) {
    float* p = out[h];
    if (p && k < a.d) p[k] = only && a.accumulate ? p[k] + v : v;
  };
  if constexpr (ROWS > 1) {                              // the sums of the sets of threads are added in order
    constexpr int WIDTH = NG * LANES * E;
    static_assert(ROWS * 2 * WIDTH * 4 <= STAGES * 2 * RB * ROW * 16);
    copies_wait<0>();                                    // the ring is free
    float* red = reinterpret_cast<float*>(ring);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int j = 0; j < H; ++j) {
        const int k = (l + i * LANES) * E + 2 * j;
        *reinterpret_cast<uint64_t*>(red + (r * 2) * WIDTH + k) = dw[i][j];
        *reinterpret_cast<uint64_t*>(red + (r * 2 + 1) * WIDTH + k) = db[i][j];
      }
    __syncthreads();
    for (int q = threadIdx.x; q < 2 * WIDTH; q += THREADS) {
      float s = 0.f;
#pragma unroll
      for (int o = 0; o < ROWS; ++o) s += red[o * 2 * WIDTH + q];
      put(q / WIDTH, q % WIDTH, s);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (l + i * LANES) * E;
        float f[E];
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 u = unpack2(h ? db[i][j] : dw[i][j]);
          f[2 * j] = u.x;
          f[2 * j + 1] = u.y;
        }
        if (!only && k < a.d) {                          // a part's row has room for whole groups
#pragma unroll
          for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(out[h] + k + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) put(h, k + j, f[j]);
        }
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
constexpr int kFinishWarps = 16;
__global__ void __launch_bounds__(32 * kFinishWarps)
bwd_finish_kernel(const float* __restrict__ part, int64_t part_ld, int n_part, int d, float* dweight, float* dbias, int accumulate) {
  pdl_wait();
  pdl_launch_dependents();
  __shared__ float red[kFinishWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.x * 32 + lane;
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  const int per = (n_part + kFinishWarps - 1) / kFinishWarps, p1 = min(n_part, (warp + 1) * per);
  float s = 0.f;
  if (k < d) {
#pragma unroll 10
    for (int p = warp * per; p < p1; ++p) s += part[((int64_t)p * 2 + blockIdx.y) * part_ld + k];
  }
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && k < d) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < kFinishWarps; ++w) s += red[w][lane];
    out[k] = accumulate ? out[k] + s : s;
  }
}

}  // namespace norm
}  // namespace flop
