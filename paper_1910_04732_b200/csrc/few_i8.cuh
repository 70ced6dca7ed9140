// 8-bit product for few tokens: the warp-level m16n8k32 instruction with the weights as rows and the tokens as columns, K dealt out in 64-long
// steps over KS of a block's eight warps, the weights read straight into registers (see gemm_few.cuh, whose form this is with bytes in place
// of bf16: a lane's 16 bytes of a row serve two instructions, K permuted alike in both operands).
//
// Bound: latency.  8 x 4096 x 1024: 3.1 us replayed, 16 x 4096 x 1024 4.4, 8 x 16384 x 4096 (67 MB of weights, 5.3 TB/s) 12.7.
// What a launch costs here is the chain of loads it waits for, so the tokens are made where they are needed: every block
// quantises (TOK_X) or requantises (TOK_H) all of them into its own shared memory, behind the request for its first weights,
// instead of a launch before it that does so once and is waited for.  A pruned matrix is two launches: tokens -> 32-bit sums of the
// first product; those -> result.  The work is repeated per block, so calls with many values of X per block take the launches
// apart (the rule is where they are launched).
// Rows of the token tile are 64 bytes modulo 128 apart, which spreads a quarter warp's 16-byte reads over all banks, and zero
// behind K; weights behind K meet those zeros.
#pragma once
#include "gemm_i8.cuh"
#include "quantized.cuh"

namespace flop {
namespace i8 {

enum { TOK_I8 = 0, TOK_BF16 = 1, TOK_F32 = 2, TOK_H = 3 };

constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps;
__host__ __device__ constexpr int few_part_stride() { return 20; }                                   // ints per token of a warp's 16-row partial tile
__host__ __device__ inline int few_stride(int K) { const int s = (K + 63) / 64; return 64 * (s | 1); }
__host__ __device__ inline size_t few_smem(int T, int K, int nt) {
  const size_t tile = (size_t)T * few_stride(K), part = (size_t)kFewWarps * 8 * nt * few_part_stride() * 4;
  return tile + part + 1024;
}

struct FewParams {
  const void* tok; int64_t ldt;                   // tokens [T, K]: 8 bits, bf16, fp32 or 32-bit sums of the product before
  const float* tok_scale;                         // TOK_I8: scale per token; TOK_H: scale per token of what went into the sums
  const float* col;                               // TOK_H: scale per column of the sums
  const int8_t* W; int64_t ldw; const float* w_scale;
  void* out; int64_t ldo;
  float* x_scale;                                 // TOK_BF16 / TOK_F32 with 32-bit sums: receives the tokens' scales
  int T, N, K;
  int vec;                                        // fp32 tokens, or sums and their column scales, start on 16 bytes in every row
};

__device__ __forceinline__ void mma_s8_16832(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of a row from k on, nothing behind K being read in the last row of a matrix
__device__ __forceinline__ uint4 load16(const int8_t* row, int k, int K, bool last) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (k + 16 <= K || (!last && k < K)) return *reinterpret_cast<const uint4*>(row + k);
  if (k < K) {
    int8_t* h = reinterpret_cast<int8_t*>(&v);
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (k + i < K) h[i] = row[k + i];
  }
  return v;
}
__device__ __forceinline__ uint32_t clip_word(uint32_t w, int left) { return left >= 4 ? w : left <= 0 ? 0u : w & (0xffffffffu >> (32 - 8 * left)); }

// ---- the tokens' tile.  Rows are dealt out over the warps, several warps to a row where there are fewer rows than warps, eight
// neighbouring values to a lane and step.  Two passes over the values (the second from L1): the largest magnitude, as the integer that its
// bits are, then the rounding.  Scale of row t ends in scale[t].
template <int TOK>
__device__ __forceinline__ void load8(const FewParams& p, const char* row, int k, float (&v)[8]) {
  if (k + 8 <= p.K && (TOK == TOK_BF16 || p.vec)) {
    if (TOK == TOK_BF16) {
      const uint4 w = *reinterpret_cast<const uint4*>(row + 2 * k);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    } else {
      const float4* at = reinterpret_cast<const float4*>(row) + k / 4;                  // (a row may have 2^30 values, 4 GB)
      const float4 x = at[0], y = at[1];
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = 0.f;
    if (k + i < p.K) {
      if (TOK == TOK_BF16) v[i] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[k + i]);
      else v[i] = reinterpret_cast<const float*>(row)[k + i];
    }
  }
}
// bf16: 127 v / amax with inv = 127 / amax rounded UP decides every value.  With v = m 2^-j u and amax = a u, 128 <= m, a < 256, a quotient that is not on
// a border is at least 1 / (a 2^(j+1)) > 1.9e-3 2^-j from it, and v inv is off by 3e-5 2^-j at most.  On a border it is only where 127 divides (2 n + 1) a:
// at v = amax / 2, where v inv is 63.5 or just above and goes to the even 64; or with a = 254, where inv is exact and so is the tie.
// (Rounded to nearest, half of those ties -- one value in 700 of normal tokens -- would have to be found and decided.)
__device__ __forceinline__ uint2 round8_bf16(const uint4& w, float inv) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    b[2 * i] = __float_as_uint(fmaf(__uint_as_float(u[i] << 16), inv, kToInt));
    b[2 * i + 1] = __float_as_uint(fmaf(__uint_as_float(u[i] & 0xffff0000u), inv, kToInt));
  }
  return bytes8(b);
}
// fp32: values within the error of a border are read again from where they are and decided exactly.
__device__ __forceinline__ uint2 round8_f32(const float (&v)[8], float inv, float amax, const float* at) {
  uint32_t b[8], near = 0;
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = fmaf(v[i], inv, kToInt), off = fabsf(fmaf(v[i], inv, kToInt - s));
    b[i] = __float_as_uint(s);
    far = fmaxf(far, off);
  }
  uint2 w = bytes8(b);
  if (far >= 0.5f - kBorder) {
#pragma unroll
    for (int i = 0; i < 8; ++i) near |= fabsf(fmaf(v[i], inv, kToInt - __uint_as_float(b[i]))) >= 0.5f - kBorder ? 1u << i : 0u;
#pragma unroll 1
    for (; near; near &= near - 1) {
      const int i = __ffs(near) - 1;
      const float x = at[i];
      const uint32_t q = (uint32_t)round_border(x, amax, (int)floorf(x * inv)) & 255u;
      const uint32_t shift = 8 * (i & 3), m = ~(255u << shift);
      if (i < 4) w.x = (w.x & m) | (q << shift);
      else w.y = (w.y & m) | (q << shift);
    }
  }
  return w;
}
// Rows whose largest magnitude is beyond 1e+-30: inv or the borders' products would leave fp32.
template <int TOK>
__device__ __noinline__ uint2 round8_wide(const char* at, int n, double amax) {
  uint32_t w[2] = {0, 0};
  for (int i = 0; i < min(n, 8); ++i) {
    const double x = TOK == TOK_F32 ? (double)reinterpret_cast<const float*>(at)[i] : (double)__bfloat162float(reinterpret_cast<const __nv_bfloat16*>(at)[i]);
    w[i >> 2] |= ((uint32_t)round_exact(x, amax) & 255u) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
// Sums times their columns' scales, in fp64 (exact as long as a sum has 29 bits): eight products from k on, 0 behind K.  They are finite
// where the scales are: `poison` (CHECK) takes 0 times every scale, and stays 0 or becomes a NaN for good.
template <bool CHECK>
__device__ __forceinline__ void products8(const FewParams& p, const char* row, int k, double (&h)[8], float& poison) {
  if (k + 8 <= p.K && p.vec) {
    const int4 x = *reinterpret_cast<const int4*>(row + 4 * k), y = *reinterpret_cast<const int4*>(row + 4 * k + 16);
    const float4 c = __ldg(reinterpret_cast<const float4*>(p.col + k)), d = __ldg(reinterpret_cast<const float4*>(p.col + k) + 1);
    h[0] = (double)x.x * (double)c.x; h[1] = (double)x.y * (double)c.y; h[2] = (double)x.z * (double)c.z; h[3] = (double)x.w * (double)c.w;
    h[4] = (double)y.x * (double)d.x; h[5] = (double)y.y * (double)d.y; h[6] = (double)y.z * (double)d.z; h[7] = (double)y.w * (double)d.w;
    if (CHECK) {
      poison = fmaf(c.w, 0.f, fmaf(c.z, 0.f, fmaf(c.y, 0.f, fmaf(c.x, 0.f, poison))));
      poison += fmaf(d.w, 0.f, fmaf(d.z, 0.f, fmaf(d.y, 0.f, d.x * 0.f)));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = k + i < p.K ? __ldg(p.col + k + i) : 0.f;
    h[i] = k + i < p.K ? (double)reinterpret_cast<const int*>(row)[k + i] * (double)s : 0.0;
    if (CHECK) poison = fmaf(s, 0.f, poison);
  }
}
__device__ __forceinline__ uint2 round8_sums(const double (&h)[8], float inv, double exact, bool careful) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = (float)h[i], s = fmaf(x, inv, kToInt);
    b[i] = __float_as_uint(s);
    if (careful) b[i] = (uint32_t)round_exact(h[i], exact);
    else if (fabsf(fmaf(x, inv, kToInt - s)) >= 0.5f - kBorderSums) b[i] = (uint32_t)round_border(h[i], exact, (int)floorf(x * inv));
  }
  return bytes8(b);
}

// warps to a row of a block that has T of them
__host__ __device__ constexpr int warps_per_row(int T) { return T > 4 ? 1 : T > 2 ? 2 : T == 2 ? 4 : 8; }

template <int TOK, int R>      // R: rows of a warp
__device__ __forceinline__ void make_tokens(const FewParams& p, int8_t* tile, int64_t stride, int limit, float* scale, float* red, int per_row) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (TOK == TOK_I8) {
    for (int t = warp; t < p.T; t += kFewWarps) {
      const int8_t* row = reinterpret_cast<const int8_t*>(p.tok) + (int64_t)t * p.ldt;
#pragma unroll 4
      for (int k = 16 * lane; k < limit; k += 512) {
        uint4 v = load16(row, k, p.K, t == p.T - 1);
        if (k + 16 > p.K) { v.x = clip_word(v.x, p.K - k); v.y = clip_word(v.y, p.K - k - 4); v.z = clip_word(v.z, p.K - k - 8); v.w = clip_word(v.w, p.K - k - 12); }
        *reinterpret_cast<uint4*>(tile + t * stride + k) = v;
      }
    }
    if (threadIdx.x < p.T) scale[threadIdx.x] = p.tok_scale ? p.tok_scale[threadIdx.x] : 1.f;
    __syncthreads();
    return;
  }
  const int sub = warp % per_row, step = 256 * per_row, k_lane = (sub * 32 + lane) * 8;
  const int rows_at_once = kFewWarps / per_row, first = warp / per_row;
  auto row_of = [&](int r) { return reinterpret_cast<const char*>(p.tok) + (int64_t)min(first + r * rows_at_once, p.T - 1) * p.ldt * (TOK == TOK_BF16 ? 2 : 4); };
  uint32_t bits[R];
#pragma unroll
  for (int r = 0; r < R; ++r) bits[r] = 0;
  int k_more = k_lane;
  if (TOK == TOK_BF16) {                                                   // two magnitudes to a word
#pragma unroll 4
    for (; k_more + 8 <= p.K; k_more += step)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint4 w = *reinterpret_cast<const uint4*>(row_of(r) + 2 * k_more);
        bits[r] = __vmaxu2(bits[r], __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
      }
#pragma unroll
    for (int r = 0; r < R; ++r) bits[r] = max(bits[r] << 16, bits[r] & 0xffff0000u);
  }
  double exact[R];
  if (TOK == TOK_H) {
    // positive doubles compare as integers: across the lanes the high words first, then the low ones among those that have the highest
#pragma unroll
    for (int r = 0; r < R; ++r) exact[r] = 0.0;
    float poison = 0.f;
#pragma unroll 1
    for (; k_more < p.K; k_more += step)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        double h[8];
        if (r == 0) products8<true>(p, row_of(r), k_more, h, poison);      // (the scales are those of every row)
        else products8<false>(p, row_of(r), k_more, h, poison);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double x = fabs(h[i]);
          if (x > exact[r]) exact[r] = x;
        }
      }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!(poison == 0.f)) exact[r] = (double)INFINITY;                   // one channel without a scale, and no token has one
      const uint32_t mine = (uint32_t)__double2hiint(exact[r]), hi = __reduce_max_sync(0xffffffffu, mine);
      const uint32_t low = __reduce_max_sync(0xffffffffu, mine == hi ? (uint32_t)__double2loint(exact[r]) : 0u);
      exact[r] = __hiloint2double((int)hi, (int)low);
    }
    if (per_row > 1) {                                                     // then R rows are one
      double* red64 = reinterpret_cast<double*>(red);
      if (lane == 0) red64[warp] = exact[0];
      __syncthreads();
      for (int w = 0; w < per_row; ++w) exact[0] = fmax(exact[0], red64[first * per_row + w]);
    }
  } else {
#pragma unroll 1
    for (; k_more < p.K; k_more += step) {
      float v[R][8];
#pragma unroll
      for (int r = 0; r < R; ++r) load8<TOK>(p, row_of(r), k_more, v[r]);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) bits[r] = max(bits[r], __float_as_uint(v[r][i]) & 0x7fffffffu);      // (infinities and NaN are the largest)
    }
    uint32_t top[R];
#pragma unroll
    for (int r = 0; r < R; ++r) top[r] = __reduce_max_sync(0xffffffffu, bits[r]);
    if (per_row > 1) {
      uint32_t* red32 = reinterpret_cast<uint32_t*>(red);
      if (lane == 0) red32[warp] = top[0];
      __syncthreads();
      for (int w = 0; w < per_row; ++w) top[0] = max(top[0], red32[first * per_row + w]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) exact[r] = (double)__uint_as_float(top[r]);
  }
  bool careful[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (!(exact[r] < (double)INFINITY)) exact[r] = (double)INFINITY;
    careful[r] = !(exact[r] < 1e30 && exact[r] > 1e-30);
  }
  if (sub == 0 && lane < R) {
    const int t = first + lane * rows_at_once;
    double e = exact[0];
#pragma unroll
    for (int r = 1; r < R; ++r) e = lane == r ? exact[r] : e;
    if (t < p.T) {
      float s = NAN;
      if (e < (double)INFINITY) s = TOK == TOK_H ? (float)((double)p.tok_scale[t] * (e * (1.0 / 127.0))) : (float)e / 127.f;
      scale[t] = s;
      if (p.x_scale && blockIdx.x == 0) p.x_scale[t] = s;
    }
  }
  float inv[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    inv[r] = exact[r] > 0.0 && exact[r] < (double)INFINITY ? (careful[r] ? 1.f : TOK == TOK_BF16 ? __fdiv_ru(127.f, (float)exact[r]) : 127.f / (float)exact[r]) : 0.f;
  }
  int k = k_lane;
  if (TOK == TOK_BF16) {                                                   // whole pieces of whole rows
    bool plain = true;
#pragma unroll
    for (int r = 0; r < R; ++r) plain &= inv[r] != 0.f && !careful[r] && first + r * rows_at_once < p.T;
    if (plain) {
#pragma unroll 4
      for (; k + 8 <= p.K; k += step)
#pragma unroll
        for (int r = 0; r < R; ++r)
          *reinterpret_cast<uint2*>(tile + (first + r * rows_at_once) * stride + k) = round8_bf16(*reinterpret_cast<const uint4*>(row_of(r) + 2 * k), inv[r]);
    }
  }
#pragma unroll 1
  for (; k < limit; k += step) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int t = first + r * rows_at_once;
      if (t >= p.T) continue;
      uint2 w = make_uint2(0, 0);
      if (k < p.K && inv[r] != 0.f) {
        const char* at = row_of(r) + (int64_t)k * (TOK == TOK_BF16 ? 2 : 4);
        float v[8];
        if (TOK != TOK_H) load8<TOK>(p, row_of(r), k, v);
        if (TOK == TOK_H) {
          double h[8];
          float unused;
          products8<false>(p, row_of(r), k, h, unused);
          w = round8_sums(h, inv[r], exact[r], careful[r]);
        } else if (careful[r]) {
          w = round8_wide<TOK>(at, p.K - k, exact[r]);
        } else if (TOK == TOK_BF16) {
          uint32_t b[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(v[i], inv[r], kToInt));
          w = bytes8(b);
        } else {
          w = round8_f32(v, inv[r], (float)exact[r], reinterpret_cast<const float*>(at));
        }
      }
      int8_t* to = tile + t * stride + k;
      if (k + 8 <= limit) *reinterpret_cast<uint2*>(to) = w;
      else
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (k + i < limit) to[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
  }
  __syncthreads();
}

// The same for a whole matrix, 8 / per_row rows to a block; columns behind `limit` of the result are left alone.
// Bound: HBM for many rows (16384 x 2048 bf16 24.4 us, 4.1 TB/s; two passes over a row, the second from L1).  For few rows, latency: a lane's values are a chain of some ten instructions each, eleven cycles apiece with two warps
// to a scheduler, so a row is spread over as many warps as leave every SM a block.
template <int TOK>
__global__ void __launch_bounds__(kFewThreads)
rows_kernel(FewParams p, int8_t* __restrict__ out, int64_t ldo, int limit, float* __restrict__ scale, int per_row) {
  __shared__ __align__(16) float red[64];
  pdl_wait();
  pdl_launch_dependents();
  const int rows = kFewWarps / per_row;
  const int64_t row0 = (int64_t)blockIdx.x * rows;
  p.tok = reinterpret_cast<const char*>(p.tok) + row0 * p.ldt * (TOK == TOK_BF16 ? 2 : 4);
  if (TOK == TOK_H) p.tok_scale += row0;
  p.T = (int)min((int64_t)rows, (int64_t)p.T - row0);
  make_tokens<TOK, 1>(p, out + row0 * ldo, ldo, limit, scale + row0, red, per_row);
}

template <int TOK, int OUT, int NT, int KS, bool EARLY>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const FewParams p) {
  constexpr int kGroups = kFewWarps / KS, kDepth = 4, S = few_part_stride();
  extern __shared__ __align__(16) unsigned char smem[];
  const int stride = few_stride(p.K);
  float* red = reinterpret_cast<float*>(smem);                            // 16 floats, 8 doubles
  float* scale = red + 64;                                                // of every token
  int8_t* tile = reinterpret_cast<int8_t*>(smem) + 1024;
  int* part = reinterpret_cast<int*>(tile + (size_t)p.T * stride);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, k_warp = warp % KS;
  const int blocks = (p.N + 16 * kGroups - 1) / (16 * kGroups);
  const int8_t* wrow[2];
  bool wlast[2];
  uint4 wv[kDepth][2];
  auto rows_of = [&](int blk) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = min((blk * kGroups + warp / KS) * 16 + 8 * i + g, p.N - 1);       // rows past the end are the last one's, and not stored
      wrow[i] = p.W + (int64_t)row * p.ldw;
      wlast[i] = row == p.N - 1;
    }
  };
  auto load_weights = [&](int s) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) wv[d][i] = load16(wrow[i], (s + d * KS) * 64 + 16 * q, p.K, wlast[i]);
  };
  int blk = blockIdx.x;
  rows_of(blk);
  if (!EARLY) pdl_wait();
  load_weights(k_warp);
  if (EARLY) pdl_wait();
  pdl_launch_dependents();
  make_tokens<TOK, NT>(p, tile, stride, stride, scale, red, warps_per_row(p.T));
  const int8_t* trow[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) trow[i] = tile + (size_t)min(8 * i + g, p.T - 1) * stride + 16 * q;
  for (; blk < blocks; blk += gridDim.x) {
    int acc[NT][4] = {};
    for (int s = k_warp; s * 64 < p.K; s += kDepth * KS) {
      if (s != k_warp) load_weights(s);
#pragma unroll
      for (int d = 0; d < kDepth; ++d) {
        const int at = (s + d * KS) * 64;
        if (at >= p.K) break;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 t = *reinterpret_cast<const uint4*>(trow[n] + at);
          mma_s8_16832(acc[n], wv[d][0].x, wv[d][1].x, wv[d][0].y, wv[d][1].y, t.x, t.y);
          mma_s8_16832(acc[n], wv[d][0].z, wv[d][1].z, wv[d][0].w, wv[d][1].w, t.z, t.w);
        }
      }
    }
    if (blk + (int)gridDim.x < blocks) { rows_of(blk + gridDim.x); load_weights(k_warp); }      // on their way while the parts are added up
    // lane (g, q) holds rows g and g + 8, tokens 8 n + 2 q and + 1
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[(warp * 8 * NT + 8 * n + 2 * q + (i & 1)) * S + g + (i >> 1) * 8] = acc[n][i];
    __syncthreads();
#pragma unroll
    for (int e = threadIdx.x; e < kGroups * 8 * NT * 8; e += kFewThreads) {      // two neighbouring columns of one token
      const int grp = e / (8 * NT * 8), t = e / 8 % (8 * NT), c = (e % 8) * 2;
      int x = 0, y = 0;
#pragma unroll
      for (int w = 0; w < KS; ++w) {
        const int2 v = *reinterpret_cast<const int2*>(part + ((grp * KS + w) * 8 * NT + t) * S + c);
        x += v.x; y += v.y;
      }
      const int n = (blk * kGroups + grp) * 16 + c;
      if (t >= p.T || n >= p.N) continue;
      if (OUT == OUT_S32) {
        int* o = reinterpret_cast<int*>(p.out) + (int64_t)t * p.ldo + n;
        o[0] = x;
        if (n + 1 < p.N) o[1] = y;
      } else {
        const float fx = (float)x * scale[t] * __ldg(p.w_scale + n), fy = n + 1 < p.N ? (float)y * scale[t] * __ldg(p.w_scale + n + 1) : 0.f;
        if (OUT == OUT_F32) {
          float* o = reinterpret_cast<float*>(p.out) + (int64_t)t * p.ldo + n;
          o[0] = fx;
          if (n + 1 < p.N) o[1] = fy;
        } else {
          __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)t * p.ldo + n;
          if (n + 1 < p.N) *reinterpret_cast<__nv_bfloat162*>(o) = __floats2bfloat162_rn(fx, fy);      // rows are 16-byte aligned, n is even
          else *o = __float2bfloat16_rn(fx);
        }
      }
    }
    if (blk + (int)gridDim.x < blocks) __syncthreads();
  }
}

}  // namespace i8
}  // namespace flop
