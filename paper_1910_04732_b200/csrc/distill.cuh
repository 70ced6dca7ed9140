// The loss of a student's logits against a teacher's top logits, and its gradient.  A compressed model is trained on what its dense
// teacher says; stored teachers keep the K largest logits of each token.
//
// Per token (row), c = 1 / temperature, p = softmax(S c) over the V words, L the words of the teacher's list (slots with an index in
// [0, V); of equal indices the first):
//     without t_lse   q = softmax over L of t c                   loss = sum_L q (log q - log p)
//     with t_lse      q = exp(t c - t_lse), r = 1 - sum_L q       loss = sum_L q (log q - log p) + r (log r - log p_rest)
// (r = 0 where the list sums to more than one or is the whole vocabulary) and p_rest is the student's mass outside L.  Every term has a -log p in it, so
// the gradient is c (n p_v - q_v) on L and c (n p_v - r p_v / p_rest) outside it, n = sum_L q + r: one, but where r is 0.
//
// The sums outside L are taken over the words outside L, not as one minus the rest: a student that agrees with its teacher leaves a
// tail of 1e-3 there, which a difference of sums near one holds to four digits.  A bit per word says which are listed (a repeated
// index shows as a bit that is already set); listed words become -inf where the row is held, so that the two passes over
// it know nothing of the list, and the K entries of the gradient are written over the zeros they leave.  Exponentials are powers of two
// relative to the largest value of their own set: nothing overflows, and a tail far below the list keeps its digits.  Sums of
// the vocabulary in fp32, of the slots in fp64 (1 - sum q cancels, and so do the two logarithms of a term), all in a fixed order.
//
// Bound: HBM for rows of thousands of words (loss alone 4096 x 128000 bf16 183 us, 5.75 TB/s), but at one exponential and some three instructions
// per element and pass the issue slots are close behind: loss and gradient of the same 562 us, 3.7 TB/s of one read and one write.
// Short rows are read once and held in registers (part_kernel): eight lanes, a warp or a block to a row, or, where rows are few, a cluster of up
// to eight blocks that exchange the maximum and sum of their parts through distributed shared memory.  With many rows, what is held is up to 4096
// pieces of 16 bytes for loss and gradient together, 512 for the loss alone and 256 for the backward call; wider rows are walked (row_kernel).
#pragma once
#include "common.cuh"

namespace flop {
namespace distill {

constexpr int kMaxSlots = 1024;
constexpr int kMaxVocab = 1 << 19;        // two bits per word in shared memory: 128 KB
constexpr double kLn2d = 0.6931471805599453;

enum { FWD = 1, BWD = 2, BOTH = 3 };

struct Args {
  const void* S; int64_t lds; int T, V;
  const float* t_logits; int64_t ldt; const int32_t* t_idx; int64_t ldi; int K;
  const float* t_lse; const float* weight;       // nullable
  float inv_tau, c; double inv_tau_d;            // 1 / temperature, log2(e) / temperature
  float* loss; float* stats;                     // FWD, BOTH (stats nullable)
  const float* stats_in; const float* dloss;     // BWD (dloss nullable)
  void* dS; int64_t ldds;                        // BWD, BOTH
  int vec;                                       // rows of S and dS start on 16 bytes
  int parts, part_pieces;                        // part_kernel: blocks per row (a cluster, but for BWD), pieces of each
};

// shared memory of one part: a bit per word in whole 16 bytes, three values per slot
__host__ __device__ inline size_t part_smem(int V, int K) { return (size_t)((V + 127) / 128) * 16 + (size_t)((3 * K + 3) / 4) * 16; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// e^x to the last bit or two of fp32, for the few values whose error would be seen in the loss
__device__ __forceinline__ float exp_of(double x) {
  const float hi = (float)x, e = expf(hi);
  return fabsf(hi) < 200.f ? e * (1.f + (float)(x - (double)hi)) : e;       // (no correction where it is infinite)
}
__device__ __forceinline__ float pow2_of(float x) { return exp_of((double)x * kLn2d); }
// log2 with the error of the fraction's logarithm: the exponent is added in fp64
__device__ __forceinline__ double log2_of(float x) {
  int e;
  const float f = frexpf(x, &e);
  return (double)log2f(f) + (double)e;
}
// log r, r = 1 - a
__device__ __forceinline__ double log_left(double a, float r) { return a < 0.5 ? (double)log1pf(-(float)a) : (double)logf(r); }
// log of the student's mass outside the list: the sum s there (relative to 2^m_rest) against the sum `top` on it (relative to 2^mc), l2a the log2 of both.
// Near zero as log1p: a difference of two logarithms of sums would be off by 1e-7 where the loss is 0.01.
__device__ __forceinline__ double log_share(float s, float m_rest, float mc, float top, double l2a) {
  const float rest = s * pow2_of(m_rest - mc);
  if (rest > 1e-30f && top < 1e30f) return rest >= top ? -(double)log1pf(top / rest) : (double)logf(rest / (rest + top));
  return ((double)m_rest - (double)mc + log2_of(s) - l2a) * kLn2d;
}
__device__ __forceinline__ float nan_max(float a, float b) { return a != a || a > b ? a : b; }
// over the W lanes (of those in `mask`) that a value belongs to
template <int W = 32, typename V, typename F>
__device__ __forceinline__ V warp_all(V v, F f, uint32_t mask = 0xffffffffu) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(mask, v, o));
  return v;
}
template <typename V> __device__ __forceinline__ V add(V a, V b) { return a + b; }
__device__ __forceinline__ float max2(float a, float b) { return fmaxf(a, b); }

// ---- pieces of a row: 16 bytes, -inf where the row has ended
template <typename T> constexpr int kPer = 16 / (int)sizeof(T);
template <typename T> __device__ __forceinline__ uint32_t neg_inf_word();
template <> __device__ __forceinline__ uint32_t neg_inf_word<float>() { return 0xff800000u; }
template <> __device__ __forceinline__ uint32_t neg_inf_word<__nv_bfloat16>() { return 0xff80ff80u; }

template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* row, int piece, int V, int vec) {
  const int at = piece * kPer<T>;
  if (vec && at + kPer<T> <= V) return __ldcs(reinterpret_cast<const uint4*>(row + at));
  uint4 v = make_uint4(neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>());
  T* h = reinterpret_cast<T*>(&v);
#pragma unroll
  for (int e = 0; e < kPer<T>; ++e)
    if (at + e < V) h[e] = row[at + e];
  return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, int piece, int V, int vec, uint4 v) {
  const int at = piece * kPer<T>;
  if (vec && at + kPer<T> <= V) { __stcs(reinterpret_cast<uint4*>(row + at), v); return; }
  const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
  for (int e = 0; e < kPer<T>; ++e)
    if (at + e < V) row[at + e] = h[e];
}
// which elements of a piece are listed
template <typename T>
__device__ __forceinline__ uint32_t listed_of(const uint32_t* bits, int piece) {
  const uint8_t* bytes = reinterpret_cast<const uint8_t*>(bits);
  if (kPer<T> == 8) return bytes[piece];
  return (bytes[piece >> 1] >> (4 * (piece & 1))) & 15u;
}
template <typename T>
__device__ __forceinline__ void hide(uint4& v, uint32_t listed) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      if (listed >> i & 1u) w[i] = 0xff800000u;
    } else {
      if (listed >> (2 * i) & 1u) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
      if (listed >> (2 * i + 1) & 1u) w[i] = (w[i] & 0xffffu) | 0xff800000u;
    }
  }
}
template <typename T>
__device__ __forceinline__ float piece_max(uint4 v) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
  if (sizeof(T) == 4) return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])), fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
  auto h = [&](int i) { return *reinterpret_cast<const __nv_bfloat162*>(&w[i]); };
  const __nv_bfloat162 m = __hmax2(__hmax2(h(0), h(1)), __hmax2(h(2), h(3)));
  return fmaxf(__low2float(m), __high2float(m));
}
// element e (compile-time after unrolling) in fp32
template <typename T>
__device__ __forceinline__ float elem(const uint4& v, int e) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
  if (sizeof(T) == 4) return __uint_as_float(w[e]);
  return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
}
template <typename T>
__device__ __forceinline__ float piece_sum(const uint4& v, float c, float m) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < kPer<T>; ++e) s += ex2(fmaf(elem<T>(v, e), c, -m));
  return s;
}
template <typename T>
__device__ __forceinline__ uint4 piece_grad(const uint4& v, float c, float m, float scale) {
  uint4 o;
  uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      w[i] = __float_as_uint(scale * ex2(fmaf(elem<T>(v, i), c, -m)));
    } else {
      const __nv_bfloat162 h = __floats2bfloat162_rn(scale * ex2(fmaf(elem<T>(v, 2 * i), c, -m)), scale * ex2(fmaf(elem<T>(v, 2 * i + 1), c, -m)));
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return o;
}

// ---- cluster
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_peer(const void* local, uint32_t rank, float a, float b) {
  uint32_t addr = (uint32_t)__cvta_generic_to_shared(local), peer;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(addr), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(peer), "f"(a), "f"(b) : "memory");
}

// One part of one row, held in registers: G threads, P pieces of 16 bytes each; G < 32 are lanes of a warp that has 32 / G rows, which go their own ways
// (masked shuffles).  16384 x 205 bf16, K = 16, loss and gradient: 10.7 us (1.5 TB/s); what bounds it is the work per row, fp64 on the slots first of all.
__host__ __device__ constexpr int part_threads(int g) { return g <= 32 ? 256 : g; }
__host__ __device__ constexpr int part_rows(int g) { return g <= 32 ? 256 / g : 1; }
template <typename T, int MODE, int G, int P>
__global__ void __launch_bounds__(part_threads(G), P > 4 || G < 32 ? 1024 / part_threads(G) : 1) part_kernel(const Args a) {
  constexpr int NW = G / 32, kGroups = part_rows(G), W = G < 32 ? G : 32;   // W: lanes that share a row
  constexpr bool kOneWarp = G <= 32;
  extern __shared__ __align__(16) unsigned char smem[];
  struct First { float t, n, x, m, s; };                // largest t, number of listed words, largest listed logit; maximum and sum outside the list
  struct Second { double a, kl; float top; };           // sum of the teacher's exponentials, of the terms, of the student's on the list
  __shared__ First first[NW > 0 ? NW : 1];
  __shared__ Second second[NW > 0 ? NW : 1];
  __shared__ float2 peer[8];
  __shared__ int s_dup[kGroups];
  const int group = kOneWarp ? threadIdx.x / G : 0, tid = kOneWarp ? threadIdx.x % G : threadIdx.x;
  const int lane = threadIdx.x & 31, warp = kOneWarp ? 0 : threadIdx.x >> 5;
  const uint32_t mask = G < 32 ? ((1u << W) - 1) << (lane & ~(W - 1)) : 0xffffffffu;
  const int64_t row = kOneWarp ? (int64_t)blockIdx.x * kGroups + group : blockIdx.x / a.parts;
  const int part = kOneWarp ? 0 : (int)(blockIdx.x % a.parts);
  const bool cluster = (MODE & FWD) && !kOneWarp && a.parts > 1;
  if (cluster) cluster_arrive();                        // completed before the first store to a peer: all of them run
  auto sync = [&] { if (kOneWarp) __syncwarp(mask); else __syncthreads(); };
  auto all = [&](auto v, auto f) { return warp_all<W>(v, f, mask); };
  const int words4 = (a.V + 127) / 128;
  unsigned char* mine = smem + (size_t)group * part_smem(a.V, a.K);
  uint32_t* bits = reinterpret_cast<uint32_t*>(mine);
  int* slot_idx = reinterpret_cast<int*>(mine + (size_t)words4 * 16);
  float* slot_t = reinterpret_cast<float*>(slot_idx + a.K);
  float* slot_x = slot_t + a.K;
  for (int i = tid; i < words4; i += G) reinterpret_cast<uint4*>(bits)[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0) s_dup[group] = 0;
  sync();
  pdl_wait();
  pdl_launch_dependents();
  if (kOneWarp && row >= a.T) return;
  const T* S = reinterpret_cast<const T*>(a.S) + row * a.lds;
  T* dS = MODE == FWD ? nullptr : reinterpret_cast<T*>(a.dS) + row * a.ldds;
  const int all_pieces = (a.V + kPer<T> - 1) / kPer<T>;
  const int lo = part * a.part_pieces, hi = min(lo + a.part_pieces, all_pieces);
  const float w = a.weight ? a.weight[row] : 1.f;
  float g = w * a.inv_tau;
  if (MODE == BWD && a.dloss) g = a.dloss[row] * g;
  bool off = MODE == BWD ? g == 0.f : w == 0.f;
  uint4 d[P];
  auto load = [&] {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lo + i * G + tid;
      d[i] = p < hi ? load_piece<T>(S, p, a.V, a.vec) : make_uint4(neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>());
    }
  };
  auto hide_listed = [&] {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lo + i * G + tid;
      const uint32_t listed = p < hi ? listed_of<T>(bits, p) : 0u;
      if (listed) hide<T>(d[i], listed);
    }
  };
  First f{-INFINITY, 0.f, -INFINITY, -INFINITY, 0.f};
  if (!off) {
    load();                                             // in flight while the list is read
    for (int j = tid; j < a.K; j += G) {
      int idx = a.t_idx[row * a.ldi + j];
      if (idx < 0 || idx >= a.V) idx = -1;
      slot_idx[j] = idx;
      if (idx < 0) continue;
      if (atomicOr(&bits[idx >> 5], 1u << (idx & 31)) >> (idx & 31) & 1u) s_dup[group] = 1;
      slot_t[j] = a.t_logits[row * a.ldt + j];
      // the backward call's parts are not ordered against one another: in place, another one's words may be gone already
      const int at = idx / kPer<T>;
      if (MODE != BWD || (at >= lo && at < hi)) slot_x[j] = to_f32(S[idx]);
    }
    sync();
    if (s_dup[group]) {                                 // rare: the first of equal indices stays
      uint32_t drop = 0;
      for (int j = tid, n = 0; j < a.K; j += G, ++n)
        if (slot_idx[j] >= 0)
          for (int i = 0; i < j; ++i)
            if (slot_idx[i] == slot_idx[j]) { drop |= 1u << n; break; }
      sync();
      for (int j = tid, n = 0; j < a.K; j += G, ++n)
        if (drop >> n & 1u) slot_idx[j] = -1;
      sync();
    }
    for (int j = tid; j < a.K; j += G)
      if (slot_idx[j] >= 0) {
        f.t = nan_max(f.t, slot_t[j]);
        f.n += 1.f;
        if (MODE & FWD) f.x = fmaxf(f.x, slot_x[j]);
      }
    f.t = all(f.t, nan_max);
    f.n = all(f.n, add<float>);
    if (MODE & FWD) {
      f.x = all(f.x, max2);
      hide_listed();
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < P; ++i) m = fmaxf(m, piece_max<T>(d[i]));
      f.m = all(m, max2);
      const float ref = f.m == -INFINITY ? 0.f : __fmul_rn(f.m, a.c);
#pragma unroll
      for (int i = 0; i < P; ++i) f.s += piece_sum<T>(d[i], a.c, ref);
      f.s = all(f.s, add<float>);
    } else {
      hide_listed();
    }
    if (NW > 1) {
      if (lane == 0) first[warp] = f;
      sync();
      First o = lane < NW ? first[lane] : First{-INFINITY, 0.f, -INFINITY, -INFINITY, 0.f};
      f.t = warp_all(o.t, nan_max);
      f.n = warp_all(o.n, add<float>);
      f.x = warp_all(o.x, max2);
      f.m = warp_all(o.m, max2);
      f.s = warp_all(o.m == -INFINITY ? o.s : o.s * pow2_of(__fmul_rn(o.m, a.c) - __fmul_rn(f.m, a.c)), add<float>);
    }
    if (cluster) {
      cluster_wait();
      if (threadIdx.x < a.parts) store_peer(&peer[part], threadIdx.x, f.m, f.s);
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      float2 o = lane < a.parts ? peer[lane] : make_float2(-INFINITY, 0.f);
      f.m = warp_all(o.x, max2);
      f.s = warp_all(o.x == -INFINITY ? o.y : o.y * pow2_of(__fmul_rn(o.x, a.c) - __fmul_rn(f.m, a.c)), add<float>);
    }
    off = f.n == 0.f || (!a.t_lse && f.t == -INFINITY);  // an empty list, or one that gives every word nothing
  } else if (cluster) {
    cluster_wait();
  }
  if (off) {
    if ((MODE & FWD) && part == 0 && tid == 0) {
      a.loss[row] = 0.f;
      if (a.stats) for (int i = 0; i < 4; ++i) a.stats[4 * row + i] = 0.f;
    }
    if (MODE & BWD)
      for (int p = lo + tid; p < hi; p += G) store_piece<T>(dS, p, a.V, a.vec, make_uint4(0, 0, 0, 0));
    return;
  }
  // the student's references in units of log 2: largest logit of all, largest outside the list
  float mc, l2all = 0.f, m_rest, l2rest;
  if (MODE & FWD) {
    m_rest = f.m == -INFINITY ? 0.f : __fmul_rn(f.m, a.c);
    mc = __fmul_rn(fmaxf(f.m, f.x), a.c);
    l2rest = log2f(f.s);
  } else {
    const float* o = a.stats_in + 4 * row;
    mc = o[0]; l2all = o[1]; m_rest = o[2]; l2rest = o[3];
  }
  // the slots: log q (up to the list's own normaliser without t_lse), q, and what they add to the sums
  const double t_ref = a.t_lse ? (double)a.t_lse[row] : (double)f.t * a.inv_tau_d;
  Second h{0.0, 0.0, 0.f};
  for (int j = tid; j < a.K; j += G) {
    if (slot_idx[j] < 0) continue;
    const double lq = (double)slot_t[j] * a.inv_tau_d - t_ref;
    const float q = exp_of(lq);
    slot_t[j] = q;
    h.a += (double)q;
    if (MODE & FWD) {
      // relative to the rounded reference that the sums are relative to
      const double lx = ((double)slot_x[j] * (double)a.c - (double)mc) * kLn2d;
      h.top += exp_of(lx);
      if (!(q <= 0.f)) h.kl += (double)q * (lq - lx);
    }
  }
  h.a = all(h.a, add<double>);
  if (MODE & FWD) { h.kl = all(h.kl, add<double>); h.top = all(h.top, add<float>); }
  if (NW > 1) {
    if (lane == 0) second[warp] = h;
    sync();
    Second o = lane < NW ? second[lane] : Second{0.0, 0.0, 0.f};
    h.a = warp_all(o.a, add<double>);
    if (MODE & FWD) { h.kl = warp_all(o.kl, add<double>); h.top = warp_all(o.top, add<float>); }
  }
  const float r = a.t_lse && f.n < (float)a.V ? (float)fmax(0.0, 1.0 - h.a) : 0.f;
  const float q_norm = a.t_lse ? 1.f : (float)(1.0 / h.a);
  const float mass = !a.t_lse || r > 0.f ? 1.f : (float)h.a;              // sum q + r
  if (MODE & FWD) {
    const double l2a = log2_of(h.top + (f.s > 0.f ? f.s * pow2_of(m_rest - mc) : f.s));
    l2all = (float)l2a;
    if (part == 0 && tid == 0) {
      double kl = h.kl + (a.t_lse ? h.a : 0.0) * l2a * kLn2d;
      if (!a.t_lse) kl = h.kl / h.a - log2_of((float)h.a) * kLn2d + l2a * kLn2d;
      if (r > 0.f) kl += (double)r * (log_left(h.a, r) - log_share(f.s, m_rest, mc, h.top, l2a));
      a.loss[row] = w * (float)kl;
      if (a.stats) { float* o = a.stats + 4 * row; o[0] = mc; o[1] = l2all; o[2] = m_rest; o[3] = l2rest; }
    }
  }
  if (MODE & BWD) {
    // outside the list: 2^(x - m_rest) times what is common to the row
    const float pull = l2rest == -INFINITY ? 0.f : g * (mass * ex2(m_rest - mc - l2all) - r * ex2(-l2rest));
    // keeps the compiler from holding the row unpacked across the reductions (123 registers instead of 80)
#pragma unroll
    for (int i = 0; i < P; ++i) asm volatile("" : "+r"(d[i].x), "+r"(d[i].y), "+r"(d[i].z), "+r"(d[i].w));
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int p = lo + i * G + tid;
      if (p < hi) store_piece<T>(dS, p, a.V, a.vec, piece_grad<T>(d[i], a.c, m_rest, pull));
    }
    sync();                                             // the zeros of the listed words are written
    for (int j = tid; j < a.K; j += G) {
      const int idx = slot_idx[j], at = idx / kPer<T>;
      if (idx >= 0 && at >= lo && at < hi) dS[idx] = from_f32<T>(g * (mass * ex2(fmaf(slot_x[j], a.c, -mc) - l2all) - slot_t[j] * q_norm));
    }
  }
}

// ---- rows that one block of G threads walks, persistent over the rows.  A thread has a batch of four 16-byte pieces in registers and the next
// one on its way, across the end of a pass and of a row.  Loss and gradient go over a row twice, the second time backwards: the last batch is
// still in registers, the rest is read again, most recent first.  What the second read costs: 1000 x 50001 bf16 64 us against 30 for the loss alone.
// (Batches kept in shared memory instead of read again: 610 to 650 us at 4096 x 128000, against 562; 64 registers do not hold that loop.)
constexpr int kBatch = 4;

__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// 2^(x c - m) of elements 2 i and 2 i + 1
template <typename T>
__device__ __forceinline__ uint64_t pair_exp(const uint4& v, int i, uint64_t c2, uint64_t neg_m2) {
  const float2 x = unpack2(fma2(pack2(elem<T>(v, 2 * i), elem<T>(v, 2 * i + 1)), c2, neg_m2));
  return pack2(ex2(x.x), ex2(x.y));
}
__device__ __forceinline__ uint32_t hmax2_word(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
template <typename T>
__device__ __forceinline__ float batch_max(const uint4 (&d)[kBatch]) {
  if (sizeof(T) == 4) {
    float m = piece_max<T>(d[0]);
#pragma unroll
    for (int i = 1; i < kBatch; ++i) m = fmaxf(m, piece_max<T>(d[i]));
    return m;
  }
  uint32_t m = hmax2_word(hmax2_word(d[0].x, d[0].y), hmax2_word(d[0].z, d[0].w));
#pragma unroll
  for (int i = 1; i < kBatch; ++i) m = hmax2_word(m, hmax2_word(hmax2_word(d[i].x, d[i].y), hmax2_word(d[i].z, d[i].w)));
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
// Named barriers of a block (0 is __syncthreads): hardware barriers of all its G threads, some of which only arrive.
__device__ __forceinline__ void bar_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int n) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(n) : "memory"); }

// shared memory: this row's list and the next one's
__host__ __device__ inline size_t row_smem(int V, int K) { return 2 * part_smem(V, K); }
constexpr int kLane = 4;                                                 // slots of a lane and round: 128 to a warp

constexpr int kBits = 1, kSums = 3, kStored = 4;                        // named barriers (kBits and kBits + 1 in turn)
struct Sums { float m, s; };                                             // maximum (logit) and sum outside the list, relative to 2^(m c)
struct Info { double q, kl; float top_ref, top, r, mass, mc, l2all, m_rest, l2rest; int empty; };      // (mass = q + r)

// The next row of a block that is looked at, from `row` on; those passed over get their loss (the list's warp) and their zeros (the others).
template <typename T, int MODE>
__device__ __forceinline__ int64_t active_from(const Args& a, int64_t row, int pieces, int tid, int threads, bool list_warp) {
  for (; row < a.T; row += gridDim.x) {
    float g = a.weight ? a.weight[row] : 1.f;
    if (MODE == BWD && a.dloss) g *= a.dloss[row];
    if (g != 0.f) break;
    if (list_warp) {
      if ((MODE & FWD) && (tid & 31) == 0) {
        a.loss[row] = 0.f;
        if (a.stats) for (int i = 0; i < 4; ++i) a.stats[4 * row + i] = 0.f;
      }
    } else if (MODE & BWD) {
      for (int p = tid; p < pieces; p += threads) store_piece<T>(reinterpret_cast<T*>(a.dS) + row * a.ldds, p, a.V, a.vec, make_uint4(0, 0, 0, 0));
    }
  }
  return row;
}
template <int MODE>
__device__ __forceinline__ float factor_of(const Args& a, int64_t row) {  // of the row's gradient
  const float g = (a.weight ? a.weight[row] : 1.f) * a.inv_tau;
  return MODE == BWD && a.dloss ? a.dloss[row] * g : g;
}

// The last warp of the block has the lists, one row ahead of the others: while they are in a row's first pass it reads the next row's list, sets
// its bits and does everything that takes only the slots; it takes the loss when the row's sums are there, and writes the K entries of the
// gradient when the others are through.  Its life is latency (index -> word -> exponentials), so loads go out four to a lane and the indices
// a row before they are used.  Barriers, in the order the other warps (M) and this one (L) meet them, row by row:
//     kBits, kBits + 1 in turn   L arrives when the row's bits are set              M waits before its first look at them
//     kSums                      both wait: M's sums and L's numbers of the row are written
//     kStored                    M arrives when the row's gradient is written       L waits before it writes the listed words and clears the bits
// The list's warp is a function of its own: in the kernel's body its registers would be taken from the other warps' (64 each).  Even so loss and
// gradient spill: 120 to 140 bytes stored and 170 to 210 loaded a thread in the kernel, 40 to 60 in this function; the loss alone spills
// nothing, the backward call at most 16 bytes.
template <typename T, int MODE, int G>
__device__ __noinline__ void row_lists(const Args& a, unsigned char* smem, Sums (*sums)[G / 32 - 1], Info* info, int64_t row, int words4, int pieces, size_t side_bytes) {
  constexpr int NW = G / 32 - 1;
  const int lane = threadIdx.x & 31;
  const T* S0 = reinterpret_cast<const T*>(a.S);
  T* dS0 = reinterpret_cast<T*>(a.dS);
  struct List { uint32_t* bits; int* idx; float *t, *x; };
  auto list_of = [&](int side) {
    List l;
    l.bits = reinterpret_cast<uint32_t*>(smem + side * side_bytes);
    l.idx = reinterpret_cast<int*>(l.bits + 4 * words4);
    l.t = reinterpret_cast<float*>(l.idx + a.K);
    l.x = l.t + a.K;
    return l;
  };
  int ahead_idx[kLane];                                                // the first 128 slots of the row after the next
  float ahead_t[kLane], ahead_lse = 0.f;
  auto load_slots = [&](int64_t row, int j0, int (&idx)[kLane], float (&t)[kLane]) {
#pragma unroll
    for (int i = 0; i < kLane; ++i) {
      const int j = j0 + 32 * i + lane;
      idx[i] = j < a.K ? a.t_idx[row * a.ldi + j] : -1;
      t[i] = j < a.K ? a.t_logits[row * a.ldt + j] : 0.f;
    }
  };
  auto load_ahead = [&](int64_t row) {
    if (row >= a.T) return;
    load_slots(row, 0, ahead_idx, ahead_t);
    if (a.t_lse) ahead_lse = a.t_lse[row];
  };
  // the list of `row` (its first slots and its lse are in ahead_*); returns the row after it, whose slots are then on their way
  auto prepare = [&](int side, int64_t row) {
    const List l = list_of(side);
    const T* S = S0 + row * a.lds;
    const double lse = a.t_lse ? (double)ahead_lse : 0.0;
    bool dup = false;
    for (int j0 = 0; j0 < a.K; j0 += 32 * kLane) {
      int idx[kLane];
      float t[kLane];
      if (j0 == 0) {
#pragma unroll
        for (int i = 0; i < kLane; ++i) { idx[i] = ahead_idx[i]; t[i] = ahead_t[i]; }
      } else {
        load_slots(row, j0, idx, t);
      }
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int j = j0 + 32 * i + lane;
        if (idx[i] < 0 || idx[i] >= a.V) idx[i] = -1;
        if (j < a.K) { l.idx[j] = idx[i]; l.t[j] = t[i]; }
        if (idx[i] >= 0) dup |= atomicOr(&l.bits[idx[i] >> 5], 1u << (idx[i] & 31)) >> (idx[i] & 31) & 1u;
      }
    }
    __syncwarp();
    bar_arrive(kBits + side, G);
    if (__any_sync(0xffffffffu, dup)) {                                // rare: the first of equal indices stays
      uint32_t drop = 0;
      for (int j = lane, n = 0; j < a.K; j += 32, ++n)
        if (l.idx[j] >= 0)
          for (int i = 0; i < j; ++i)
            if (l.idx[i] == l.idx[j]) { drop |= 1u << n; break; }
      __syncwarp();
      for (int j = lane, n = 0; j < a.K; j += 32, ++n)
        if (drop >> n & 1u) l.idx[j] = -1;
      __syncwarp();
    }
    float mt = -INFINITY, mx = -INFINITY;
    int n = 0;
    for (int j0 = 0; j0 < a.K; j0 += 32 * kLane) {
      float x[kLane];
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int j = j0 + 32 * i + lane, idx = j < a.K ? l.idx[j] : -1;
        x[i] = idx >= 0 ? to_f32(S[idx]) : -INFINITY;
        if (idx >= 0) { mt = nan_max(mt, l.t[j]); ++n; }
      }
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int j = j0 + 32 * i + lane;
        if (j < a.K) l.x[j] = x[i];
        mx = fmaxf(mx, x[i]);
      }
    }
    const int64_t after = active_from<T, MODE>(a, row + gridDim.x, pieces, lane, 32, true);
    load_ahead(after);
    mt = warp_all(mt, nan_max); mx = warp_all(mx, max2);
    n = __reduce_add_sync(0xffffffffu, n);
    const double t_ref = a.t_lse ? lse : (double)mt * a.inv_tau_d;
    // the student's exponentials on the list relative to the largest there
    const float ref = !(MODE & FWD) || mx == -INFINITY ? 0.f : __fmul_rn(mx, a.c);
    float top = 0.f;
    double sum_q = 0.0, kl = 0.0;
    for (int j = lane; j < a.K; j += 32) {
      if (l.idx[j] < 0) continue;
      const double lq = (double)l.t[j] * a.inv_tau_d - t_ref;
      const float q = exp_of(lq);
      l.t[j] = q;
      sum_q += (double)q;
      if (MODE & FWD) {
        const double lx = ((double)l.x[j] * (double)a.c - (double)ref) * kLn2d;
        const float e = exp_of(lx);
        l.x[j] = e;
        top += e;
        if (!(q <= 0.f)) kl += (double)q * (lq - lx);
      }
    }
    sum_q = warp_all(sum_q, add<double>);
    if (MODE & FWD) { kl = warp_all(kl, add<double>); top = warp_all(top, add<float>); }
    if (lane == 0) {
      Info& o = info[side];
      o.q = sum_q; o.kl = kl; o.top_ref = ref; o.top = top;
      o.r = a.t_lse && n < a.V ? (float)fmax(0.0, 1.0 - sum_q) : 0.f;
      o.mass = !a.t_lse || o.r > 0.f ? 1.f : (float)sum_q;
      o.empty = n == 0 || (!a.t_lse && mt == -INFINITY);               // an empty list, or one that gives every word nothing
      if (MODE == BWD) { const float* st = a.stats_in + 4 * row; o.mc = st[0]; o.l2all = st[1]; o.m_rest = st[2]; o.l2rest = st[3]; }
    }
    __syncwarp();
    return after;
  };
  int side = 0;
  load_ahead(row);
  int64_t next = prepare(0, row);
  for (;;) {
    // the loss alone has one pass to hide the next list behind, loss and gradient rather the second
    int64_t after = next;
    if (MODE != BOTH && next < a.T) after = prepare(side ^ 1, next);
    bar_sync(kSums, G);
    const Info o = info[side];
    float all_inv = 0.f;
    const float q_norm = a.t_lse ? 1.f : (float)(1.0 / o.q);
    if (MODE & FWD) {
      const Sums u = lane < NW ? sums[side][lane] : Sums{-INFINITY, 0.f};
      const float m = warp_all(u.m, max2), m_rest = m == -INFINITY ? 0.f : __fmul_rn(m, a.c);
      const float s = warp_all(u.m == -INFINITY ? u.s : u.s * pow2_of(__fmul_rn(u.m, a.c) - m_rest), add<float>);
      // relative to the larger reference
      const float mc = o.top > 0.f || o.top != o.top ? fmaxf(o.top_ref, m == -INFINITY ? o.top_ref : m_rest) : m_rest;
      // (a list that the student rules out whole has no reference: 0 at one far above the rest's would be 0 times infinity)
      const float to_mc = o.top == 0.f ? 0.f : pow2_of(o.top_ref - mc);
      const float on = o.top * to_mc;
      const float all = on + (s > 0.f ? s * pow2_of(m_rest - mc) : s);
      all_inv = o.mass * to_mc / all;
      if (lane == 0) {
        const double l2a = log2_of(all);
        // the terms' logarithms are relative to the list's reference
        const double log_all = (l2a + (double)mc - (double)o.top_ref) * kLn2d;
        double v = a.t_lse ? o.kl + o.q * log_all : o.kl / o.q - log2_of((float)o.q) * kLn2d + log_all;
        if (o.r > 0.f) v += (double)o.r * (log_left(o.q, o.r) - log_share(s, m_rest, mc, on, l2a));
        a.loss[row] = o.empty ? 0.f : (a.weight ? a.weight[row] : 1.f) * (float)v;
        if (a.stats) { float* st = a.stats + 4 * row; st[0] = mc; st[1] = (float)l2a; st[2] = m_rest; st[3] = log2f(s); }
      }
    }
    if (MODE == BOTH && next < a.T) after = prepare(side ^ 1, next);
    // what is left of a row when its gradient is written: the listed words, and their bits
    const List l = list_of(side);
    if (MODE & BWD) {
      const float g = factor_of<MODE>(a, row);
      bar_sync(kStored, G);
      for (int j = lane; j < a.K; j += 32)
        if (l.idx[j] >= 0 && !o.empty) {
          const float p = MODE == BWD ? o.mass * ex2(fmaf(l.x[j], a.c, -o.mc) - o.l2all) : l.x[j] * all_inv;
          dS0[row * a.ldds + l.idx[j]] = from_f32<T>(g * (p - l.t[j] * q_norm));
        }
    }
    for (int j = lane; j < a.K; j += 32)
      if (l.idx[j] >= 0) atomicAnd(&l.bits[l.idx[j] >> 5], ~(1u << (l.idx[j] & 31)));
    __syncwarp();
    if (next >= a.T) break;
    row = next;
    next = after;
    side ^= 1;
  }
}

template <typename T, int MODE, int G>
__global__ void __launch_bounds__(G, 1024 / G) row_kernel(const __grid_constant__ Args a) {
  constexpr int M = G - 32, NW = M / 32;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Sums sums[2][NW];
  __shared__ Info info[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words4 = (a.V + 127) / 128, pieces = (a.V + kPer<T> - 1) / kPer<T>;
  const size_t side_bytes = part_smem(a.V, a.K);
  for (size_t i = tid; i < 2 * side_bytes / 16; i += G) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  const T* S0 = reinterpret_cast<const T*>(a.S);
  T* dS0 = reinterpret_cast<T*>(a.dS);
  int64_t row = active_from<T, MODE>(a, blockIdx.x, pieces, tid, M, warp == NW);
  if (row >= a.T) return;
  if (warp == NW) {
    row_lists<T, MODE, G>(a, smem, sums, info, row, words4, pieces, side_bytes);
    return;
  }

  // ------------------------------------------------------------------------------------ the vocabulary
  const int batches = (pieces + M * kBatch - 1) / (M * kBatch);
  const int whole = a.vec ? a.V / (kPer<T> * M * kBatch) : 0;            // batches whose pieces are all there
  uint4 d[kBatch], ahead[kBatch];
  auto load = [&](uint4 (&to)[kBatch], const T* S, int b) {
    if (b < whole) {
      const uint4* p = reinterpret_cast<const uint4*>(S) + b * kBatch * M + tid;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) to[i] = p[i * M];
    } else {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int p = (b * kBatch + i) * M + tid;
        to[i] = p < pieces ? load_piece<T>(S, p, a.V, a.vec) : make_uint4(neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>(), neg_inf_word<T>());
      }
    }
  };
  int side = 0;
  auto hide_listed = [&](int b) {
    const uint8_t* at = smem + side * side_bytes;
    uint32_t l[kBatch], any = 0;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int p = (b * kBatch + i) * M + tid;
      l[i] = 0;
      if (b < whole || p < pieces) l[i] = kPer<T> == 8 ? at[p] : (at[p >> 1] >> (4 * (tid & 1))) & 15u;      // (M is even)
      any |= l[i];
    }
    if (any) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (l[i]) hide<T>(d[i], l[i]);
    }
  };
  const uint64_t c2 = pack2(a.c, a.c);
  load(ahead, S0 + row * a.lds, 0);
  for (;;) {
    const T* S = S0 + row * a.lds;
    const int64_t next = active_from<T, MODE>(a, row + gridDim.x, pieces, tid, M, false);
    const T* S_next = next < a.T ? S0 + next * a.lds : nullptr;
    bar_sync(kBits + side, G);
    float m = -INFINITY;
    if (MODE & FWD) {
      // first pass: maximum and sum outside the list, kept relative to the maximum so far
      float ref = 0.f;
      uint64_t s2 = pack2(0.f, 0.f), neg_ref2 = pack2(0.f, 0.f);
      for (int b = 0; b < batches; ++b) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) d[i] = ahead[i];
        if (b + 1 < batches) load(ahead, S, b + 1);
        else if (MODE == BOTH && batches > 1) load(ahead, S, batches - 2);
        else if (S_next) load(ahead, S_next, 0);
        hide_listed(b);
        const float mv = batch_max<T>(d);
        if (mv > m) {
          const float to = __fmul_rn(mv, a.c), by = ex2(m == -INFINITY ? -INFINITY : ref - to);
          s2 = mul2(s2, pack2(by, by));
          m = mv; ref = to;
          neg_ref2 = pack2(-to, -to);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          uint64_t e = pair_exp<T>(d[i], 0, c2, neg_ref2);
#pragma unroll
          for (int j = 1; j < kPer<T> / 2; ++j) e = add2(e, pair_exp<T>(d[i], j, c2, neg_ref2));
          s2 = add2(s2, e);
        }
      }
      const float2 both = unpack2(s2);
      float s = both.x + both.y;
      const float mw = warp_all(m, max2);
      s = warp_all(m == -INFINITY ? s : s * ex2(ref - __fmul_rn(mw, a.c)), add<float>);
      if (lane == 0) sums[side][warp] = Sums{mw, s};
    }
    bar_sync(kSums, G);
    if (MODE & BWD) {
      // second pass: outside the list 2^(x - m_rest) times what is common to the row
      const Info& o = info[side];
      const float g = factor_of<MODE>(a, row), r = o.r;
      float m_rest, pull;
      if (MODE == BWD) {
        m_rest = o.m_rest;
        pull = o.l2rest == -INFINITY ? 0.f : g * (o.mass * ex2(m_rest - o.mc - o.l2all) - r * ex2(-o.l2rest));
      } else {
        const Sums u = lane < NW ? sums[side][lane] : Sums{-INFINITY, 0.f};
        const float ma = warp_all(u.m, max2);
        m_rest = ma == -INFINITY ? 0.f : __fmul_rn(ma, a.c);
        const float s = warp_all(u.m == -INFINITY ? u.s : u.s * ex2(__fmul_rn(u.m, a.c) - m_rest), add<float>);
        // mass / (all words' sum) - r / (the rest's), both relative to the rest's maximum; a list far above it makes the first one 0
        pull = s == 0.f ? 0.f : g * (o.mass / (s + (o.top == 0.f ? 0.f : o.top * ex2(o.top_ref - m_rest))) - r / s);
      }
      const bool empty = o.empty;
      T* dS = dS0 + row * a.ldds;
      const uint64_t neg_ref2 = pack2(-m_rest, -m_rest), pull2 = pack2(pull, pull);
      // with a first pass before it, backwards: what was read last is here, in L1 or in L2
      for (int n = 0; n < batches; ++n) {
        const int b = MODE == BOTH ? batches - 1 - n : n;
        if (MODE == BWD || n > 0) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) d[i] = ahead[i];
          if (n + 1 < batches) load(ahead, S, MODE == BOTH ? b - 1 : b + 1);
          else if (S_next) load(ahead, S_next, 0);
          hide_listed(b);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          uint4 o4;
          uint32_t* ow = reinterpret_cast<uint32_t*>(&o4);
#pragma unroll
          for (int j = 0; j < kPer<T> / 2; ++j) {
            const float2 e = unpack2(mul2(pair_exp<T>(d[i], j, c2, neg_ref2), pull2));
            if (sizeof(T) == 4) {
              ow[2 * j] = __float_as_uint(e.x); ow[2 * j + 1] = __float_as_uint(e.y);
            } else {
              const __nv_bfloat162 hh = __floats2bfloat162_rn(e.x, e.y);
              ow[j] = *reinterpret_cast<const uint32_t*>(&hh);
            }
          }
          if (empty) o4 = make_uint4(0, 0, 0, 0);
          const int p = (b * kBatch + i) * M + tid;
          if (b < whole) __stcs(reinterpret_cast<uint4*>(dS) + p, o4);
          else if (p < pieces) store_piece<T>(dS, p, a.V, a.vec, o4);
        }
      }
      bar_arrive(kStored, G);
    }
    if (next >= a.T) break;
    row = next;
    side ^= 1;
  }
}

}  // namespace distill
}  // namespace flop
