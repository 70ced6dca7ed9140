// Rows of tokens in pieces.  A group is eight columns (16 bytes of bf16, 32 of fp32), what one block of the generator serves; a unit is 16 bytes, what a thread copies,
// loads and stores at once.  A row's last group and unit may hold fewer columns.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "common.cuh"
#include "pairs.cuh"

namespace flop {

template <typename T> struct Raw8;                              // a group as it lies in memory
template <> struct Raw8<__nv_bfloat16> { uint4 q[1]; };
template <> struct Raw8<float> { uint4 q[2]; };

// The group of `n` columns at p (n > 8: eight, n <= 0: none).  vec: rows start on 16 bytes.  inner: another row follows, so the
// 16-byte piece that holds the row's end may be read whole.  Columns past n are not defined (unpack8 clears them).
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n, bool vec, bool inner) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r) / 16); ++i) r.q[i] = make_uint4(0, 0, 0, 0);
  if (vec && (n >= 8 || (inner && n > 0))) {
    r.q[0] = *reinterpret_cast<const uint4*>(p);
    if (sizeof(T) == 4 && n > 4) r.q[sizeof(r) / 16 - 1] = *(reinterpret_cast<const uint4*>(p) + 1);
  } else if (n > 0) {
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : from_f32<T>(0.f);
    memcpy(&r, v, sizeof(r));
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, int n, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    memcpy(v, &r, 32);
  } else {
    const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  if (n < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
    memcpy(&r, v, 32);
  } else {
    __nv_bfloat162 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    memcpy(&r, w, 16);
  }
  return r;
}

// Columns from n on are left untouched.
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r, int n, bool vec) {
  if (vec && n >= 8) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r) / 16); ++i) *(reinterpret_cast<uint4*>(p) + i) = r.q[i];
  } else {
    T v[8];
    memcpy(v, &r, sizeof(r));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = v[j];
  }
}

// ---- units: 16 bytes of a row
template <typename T> constexpr int kUnit = 16 / (int)sizeof(T);      // columns of a unit
template <typename T> constexpr int kPairs = kUnit<T> / 2;

// Asynchronous copies to shared memory, which a thread reads back itself once its own have arrived.
__device__ __forceinline__ void copy_async16(void* to, const void* from, int bytes) {      // zeros behind `bytes`
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async4(void* to, const void* from, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <typename T>
__device__ __forceinline__ void copy_unit(uint4* to, const T* from, int n, bool vec) {     // n columns (<= 0: none), zeros behind them
  if (sizeof(T) == 2 || vec) {
    copy_async16(to, from, min(max(n, 0), kUnit<T>) * (int)sizeof(T));
  } else {
#pragma unroll
    for (int j = 0; j < kUnit<T>; ++j) copy_async4(reinterpret_cast<T*>(to) + j, from + j, j < n ? 4 : 0);
  }
}

// Columns of the unit at p that are there (n <= 0: none), zeros behind them.  inner: another row follows, so the unit that holds a row's end may be read whole
// (what is behind the end is not cleared then).
template <typename T>
__device__ __forceinline__ uint4 load_unit(const T* p, int n, bool vec, bool inner) {
  uint4 q = make_uint4(0, 0, 0, 0);
  if ((sizeof(T) == 2 || vec) && (n >= kUnit<T> || (inner && n > 0))) {
    q = *reinterpret_cast<const uint4*>(p);
  } else if (n > 0) {
    T v[kUnit<T>];
#pragma unroll
    for (int j = 0; j < kUnit<T>; ++j) v[j] = j < n ? p[j] : from_f32<T>(0.f);
    memcpy(&q, v, 16);
  }
  return q;
}
template <typename T>
__device__ __forceinline__ void unpack_unit(const uint4& q, uint64_t (&v)[kPairs<T>]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < kPairs<T>; ++j) {
    if constexpr (sizeof(T) == 2) v[j] = pack2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
    else v[j] = pack2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack_unit(const uint64_t (&v)[kPairs<T>]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < kPairs<T>; ++j) {
    const float2 u = unpack2(v[j]);
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(u.x, u.y);
      memcpy(&w[j], &h, 4);
    } else {
      w[2 * j] = __float_as_uint(u.x);
      w[2 * j + 1] = __float_as_uint(u.y);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store_unit(T* p, const uint4& q, int n, bool vec) {
  if ((sizeof(T) == 2 || vec) && n >= kUnit<T>) {
    *reinterpret_cast<uint4*>(p) = q;
  } else {
    T v[kUnit<T>];
    memcpy(v, &q, 16);
#pragma unroll
    for (int j = 0; j < kUnit<T>; ++j)
      if (j < n) p[j] = v[j];
  }
}

}  // namespace flop
