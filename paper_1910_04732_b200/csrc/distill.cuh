// The loss of a student's logits against a teacher's top logits, and its gradient.  A compressed model is trained on what its dense
// teacher says; stored teachers keep the K largest logits of each token.
//
// Per token (row), c = 1 / temperature, p = softmax(S c) over the V words, L the words of the teacher's list (slots with an index in
// [0, V); of equal indices the first):
//     without t_lse   q = softmax over L of t c                   loss = sum_L q (log q - log p)
//     with t_lse      q = exp(t c - t_lse), r = 1 - sum_L q       loss = sum_L q (log q - log p) + r (log r - log p_rest)
// where p_rest is the student's mass outside L.  Gradient: c (p_v - q_v) on L and c (p_v - r p_v / p_rest) outside it.
//
// The sums outside L are taken over the words outside L, not as one minus the rest: a student that agrees with its teacher leaves a
// tail of 1e-3 there, which a difference of sums near one holds to four digits.  A bit per word says which are listed; a repeated
// index shows as a bit that is already set.  Everything is held in units of log 2, relative to the largest value of its own set, so
// nothing overflows and a tail far below the list keeps its digits.  Sums in fp32, in a fixed order.
#pragma once
#include "common.cuh"

namespace flop {
namespace distill {

constexpr int kMaxSlots = 1024;
constexpr int kMaxVocab = 1 << 20;        // a bit per word in shared memory: 128 KB
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum { FWD = 1, BWD = 2, BOTH = 3 };

struct Args {
  const void* S; int64_t lds; int V;
  const float* t_logits; int64_t ldt; const int32_t* t_idx; int64_t ldi; int K;
  const float* t_lse; const float* weight;       // nullable
  float inv_tau, c;                              // 1 / temperature, log2(e) / temperature
  float* loss; float* stats;                     // FWD, BOTH (stats nullable)
  const float* stats_in; const float* dloss;     // BWD (dloss nullable)
  void* dS; int64_t ldds;                        // BWD, BOTH
  int vec;                                       // rows of S and dS start on 16 bytes
};

constexpr int kThreads = 256;

// Value over the block, the warps' results joined in warp order; every thread gets it.  `red`: 32 floats.
template <typename F>
__device__ __forceinline__ float block_reduce(float v, float* red, F f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < (int)blockDim.x / 32; ++w) v = f(v, red[w]);
  return v;
}
__device__ __forceinline__ float fadd(float a, float b) { return a + b; }
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float nan_max(float a, float b) { return a != a || a > b ? a : b; }

template <typename T, int MODE>
__global__ void __launch_bounds__(kThreads) row_kernel(const Args a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float red[32];
  __shared__ int s_dup;
  const int words = (a.V + 31) / 32;
  uint32_t* bits = reinterpret_cast<uint32_t*>(smem);
  int* slot_idx = reinterpret_cast<int*>(bits + words);
  float* slot_t = reinterpret_cast<float*>(slot_idx + a.K);      // teacher's logit, then q
  float* slot_x = slot_t + a.K;                                  // student's logit
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  const T* S = reinterpret_cast<const T*>(a.S) + row * a.lds;
  T* dS = MODE == FWD ? nullptr : reinterpret_cast<T*>(a.dS) + row * a.ldds;
  const float w = a.weight ? a.weight[row] : 1.f;
  float g = w * a.inv_tau;
  if (MODE == BWD && a.dloss) g = a.dloss[row] * g;
  bool off = MODE == BWD ? g == 0.f : w == 0.f;
  for (int i = tid; i < words; i += kThreads) bits[i] = 0;
  if (tid == 0) s_dup = 0;
  __syncthreads();
  float mt = -INFINITY, n_listed = 0.f;
  if (!off) {
    for (int j = tid; j < a.K; j += kThreads) {
      int idx = a.t_idx[row * a.ldi + j];
      if (idx < 0 || idx >= a.V) idx = -1;
      slot_idx[j] = idx;
      if (idx < 0) continue;
      if (atomicOr(&bits[idx >> 5], 1u << (idx & 31)) >> (idx & 31) & 1u) s_dup = 1;
      slot_t[j] = a.t_logits[row * a.ldt + j];
      slot_x[j] = to_f32(S[idx]);
    }
    __syncthreads();
    if (s_dup) {            // rare: the first of equal indices stays
      uint32_t drop = 0;
      for (int j = tid, n = 0; j < a.K; j += kThreads, ++n)
        for (int i = 0; i < j; ++i)
          if (slot_idx[i] == slot_idx[j]) { drop |= 1u << n; break; }
      __syncthreads();
      for (int j = tid, n = 0; j < a.K; j += kThreads, ++n)
        if (drop >> n & 1u) slot_idx[j] = -1;
      __syncthreads();
    }
    for (int j = tid; j < a.K; j += kThreads)
      if (slot_idx[j] >= 0) { mt = nan_max(mt, slot_t[j]); n_listed += 1.f; }
    mt = block_reduce(mt, red, nan_max);
    n_listed = block_reduce(n_listed, red, fadd);
    off = n_listed == 0.f || (!a.t_lse && mt == -INFINITY);      // an empty list, or one that gives every word nothing
  }
  if (off) {
    if (MODE & FWD) {
      if (tid == 0) {
        a.loss[row] = 0.f;
        if (a.stats) for (int i = 0; i < 4; ++i) a.stats[4 * row + i] = 0.f;
      }
    }
    if (MODE & BWD)
      for (int v = tid; v < a.V; v += kThreads) dS[v] = from_f32<T>(0.f);
    return;
  }
  // the teacher: log2 q and q of every slot
  float lt = 0.f;
  if (!a.t_lse) {
    float s = 0.f;
    for (int j = tid; j < a.K; j += kThreads)
      if (slot_idx[j] >= 0) s += exp2f((slot_t[j] - mt) * a.c);
    lt = log2f(block_reduce(s, red, fadd));
  } else {
    const float lse = a.t_lse[row];
    mt = 0.f;
    for (int j = tid; j < a.K; j += kThreads)
      if (slot_idx[j] >= 0) slot_t[j] = fmaf(slot_t[j], a.inv_tau, -lse);
  }
  auto log2q = [&](int j) { return a.t_lse ? slot_t[j] * kLog2e : fmaf(slot_t[j] - mt, a.c, -lt); };
  float Q = 0.f;
  for (int j = tid; j < a.K; j += kThreads)
    if (slot_idx[j] >= 0) Q += exp2f(log2q(j));
  Q = block_reduce(Q, red, fadd);
  const float r = a.t_lse && n_listed < (float)a.V ? fmaxf(0.f, 1.f - Q) : 0.f;
  // the student: largest value and sum of exponentials outside the list and over all words
  float mc, l2all, m_rest, l2rest;
  if (MODE & FWD) {
    float m = -INFINITY, mx = -INFINITY;
    for (int v = tid; v < a.V; v += kThreads)
      if (!(bits[v >> 5] >> (v & 31) & 1u)) m = fmaxf(m, to_f32(S[v]));
    m = block_reduce(m, red, fmax2);
    m_rest = m == -INFINITY ? 0.f : m * a.c;
    float s = 0.f;
    for (int v = tid; v < a.V; v += kThreads)
      if (!(bits[v >> 5] >> (v & 31) & 1u)) s += exp2f(fmaf(to_f32(S[v]), a.c, -m_rest));
    s = block_reduce(s, red, fadd);
    for (int j = tid; j < a.K; j += kThreads)
      if (slot_idx[j] >= 0) mx = fmaxf(mx, slot_x[j]);
    mx = fmaxf(m, block_reduce(mx, red, fmax2));
    mc = mx * a.c;
    float st = 0.f;
    for (int j = tid; j < a.K; j += kThreads)
      if (slot_idx[j] >= 0) st += exp2f(fmaf(slot_x[j], a.c, -mc));
    st = block_reduce(st, red, fadd);
    l2rest = log2f(s);
    l2all = log2f(st + (s > 0.f ? s * exp2f(m_rest - mc) : s));
    float kl = 0.f;
    for (int j = tid; j < a.K; j += kThreads) {
      if (slot_idx[j] < 0) continue;
      const float lq = log2q(j), q = exp2f(lq);
      if (!(q <= 0.f)) kl += q * (lq - (fmaf(slot_x[j], a.c, -mc) - l2all));
    }
    kl = block_reduce(kl, red, fadd);
    if (r > 0.f) kl += r * (log2f(r) - (m_rest - mc + l2rest - l2all));
    if (tid == 0) {
      a.loss[row] = w * (kl * kLn2);
      if (a.stats) { float* o = a.stats + 4 * row; o[0] = mc; o[1] = l2all; o[2] = m_rest; o[3] = l2rest; }
    }
  } else {
    const float* o = a.stats_in + 4 * row;
    mc = o[0]; l2all = o[1]; m_rest = o[2]; l2rest = o[3];
  }
  if (MODE & BWD) {
    // outside the list: 2^(x - m_rest) times what is common to the row
    const float pull = l2rest == -INFINITY ? 0.f : g * (exp2f(m_rest - mc - l2all) - r * exp2f(-l2rest));
    for (int v = tid; v < a.V; v += kThreads) {
      if (bits[v >> 5] >> (v & 31) & 1u) continue;
      dS[v] = from_f32<T>(pull * exp2f(fmaf(to_f32(S[v]), a.c, -m_rest)));
    }
    for (int j = tid; j < a.K; j += kThreads) {
      if (slot_idx[j] < 0) continue;
      dS[slot_idx[j]] = from_f32<T>(g * (exp2f(fmaf(slot_x[j], a.c, -mc) - l2all) - exp2f(log2q(j))));
    }
  }
}

}  // namespace distill
}  // namespace flop
