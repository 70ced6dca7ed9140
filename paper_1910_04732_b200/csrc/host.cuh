// Host-side helpers of the C entry points: error returns, launches, argument checks, workspace layout.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <utility>

#include "../../include/flop.h"
#include "per_device.cuh"

namespace flop {

// FLOP_DEBUG=1 in the environment prints the failing CUDA call to stderr.
inline bool debug_on() {
  static int v = -1;
  if (v < 0) { const char* e = getenv("FLOP_DEBUG"); v = (e && e[0] && e[0] != '0') ? 1 : 0; }
  return v == 1;
}
#define FLOP_CUDA(expr)                                                                           \
  do {                                                                                            \
    cudaError_t e__ = (expr);                                                                     \
    if (e__ != cudaSuccess) {                                                                     \
      if (debug_on()) fprintf(stderr, "[flop] %s:%d: %s -> %s\n", __FILE__, __LINE__, #expr, cudaGetErrorString(e__)); \
      cudaGetLastError();                                                                         \
      return FLOP_ERR_CUDA;                                                                       \
    }                                                                                             \
  } while (0)
#define FLOP_TRY(expr)              \
  do {                              \
    int s__ = (expr);               \
    if (s__ != FLOP_OK) return s__; \
  } while (0)


// Tuning switches.  A library built with -DFLOP_TUNING reads them once from the environment (they exist to
// compare variants on one machine); the normal build takes the defaults below and reads nothing but FLOP_DEBUG.
//   FLOP_NO_PDL=1          launch without programmatic dependent launch
//   FLOP_TC_BN / FLOP_TC_STAGES / FLOP_TC_CTA2 (1 force pairs, 2 forbid)     tile shape of single GEMMs
//   FLOP_TC_GROUP_BN / FLOP_TC_GROUP_CTA2, FLOP_TC_WGRAD_BN / FLOP_TC_WGRAD_CTA2   tile shape of grouped launches
//   FLOP_NO_TMA_STORE=1    bf16 output tiles by per-thread stores    FLOP_NO_SCHED=1   round-robin tile order
//   FLOP_NO_FEW=1          few-token forward kernel off
//   FLOP_STAGE_MERGE=0     backward in three launches per stage instead of two shared ones
//   FLOP_GATHER_PIPE=0     plain P gather kernel                     FLOP_NO_CHAIN=1   chained calls run unchained
//   FLOP_CHAIN_STAGES=2    chained calls put dependent products in ONE launch (default 1: a launch per stage)
//   FLOP_SCHED_EPI=c       per-tile fixed cost (SM cycles) in the tile schedule's cost model instead of 400 + 4 bn
struct Tuning {
  int no_pdl = 0, tc_bn = 0, tc_stages = 0, tc_cta2 = 0, no_tma_store = 0, no_sched = 0, group_bn = 0, group_cta2 = 0,
      wgrad_bn = 0, wgrad_cta2 = 0, no_few = 0, stage_merge = 1, gather_pipe = 1, no_chain = 0, chain_stages = 1, sched_epi = 0;
};
inline const Tuning& tuning() {
  static const Tuning t = [] {
    Tuning v;
#ifdef FLOP_TUNING
    auto get = [](const char* name, int dflt) { const char* e = getenv(name); return e ? atoi(e) : dflt; };
    v.no_pdl = get("FLOP_NO_PDL", 0); v.tc_bn = get("FLOP_TC_BN", 0); v.tc_stages = get("FLOP_TC_STAGES", 0);
    v.tc_cta2 = get("FLOP_TC_CTA2", 0); v.no_tma_store = get("FLOP_NO_TMA_STORE", 0); v.no_sched = get("FLOP_NO_SCHED", 0);
    v.group_bn = get("FLOP_TC_GROUP_BN", 0); v.group_cta2 = get("FLOP_TC_GROUP_CTA2", 0); v.wgrad_bn = get("FLOP_TC_WGRAD_BN", 0);
    v.wgrad_cta2 = get("FLOP_TC_WGRAD_CTA2", 0); v.no_few = get("FLOP_NO_FEW", 0);
    v.stage_merge = get("FLOP_STAGE_MERGE", 1); v.gather_pipe = get("FLOP_GATHER_PIPE", 1); v.no_chain = get("FLOP_NO_CHAIN", 0);
    v.chain_stages = get("FLOP_CHAIN_STAGES", 1); v.sched_epi = get("FLOP_SCHED_EPI", 0);
#endif
    return v;
  }();
  return t;
}

// Every kernel goes through here: programmatic dependent launch lets a kernel's prologue overlap
// the tail of its predecessor on the stream (the kernels call griddepcontrol.wait before they
// touch global memory).
inline bool pdl_on() { return !tuning().no_pdl; }
template <typename... KArgs, typename... Args>
inline void launch_k(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_on() ? 1 : 0;
  cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);   // errors are picked up by cudaGetLastError()
}

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int64_t round_up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A caller's buffer, from its first byte to one past its last (nothing when the pointer is null).  A launch whose blocks read what
// another of its blocks writes needs its outputs apart from its inputs; a sequence of launches often does not, so a call
// whose buffers overlap keeps the sequence.
struct Span {
  uintptr_t lo = 0, hi = 0;
  Span() = default;
  Span(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t elem) {
    if (!p || rows <= 0 || cols <= 0) return;
    lo = reinterpret_cast<uintptr_t>(p);
    hi = lo + (size_t)((rows - 1) * ld + cols) * elem;
  }
  bool meets(const Span& o) const { return lo < o.hi && o.lo < hi; }
};
inline bool valid_dt(int dt) { return dt == FLOP_F32 || dt == FLOP_BF16; }
inline size_t elt(int dt) { return dt == FLOP_BF16 ? 2 : 4; }
inline bool valid_hc(const flop_hc_params_t& hc) { return hc.beta > 0.f && hc.gamma < 0.f && hc.zeta > 1.f; }

// Per-device state (function attributes already set, SM count, built-in scratch address) is indexed by the
// current device, so that a process that drives several GPUs configures each of them.
inline int current_device() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return -1; }
  return (dev >= 0 && dev < kMaxDevices) ? dev : -1;
}
// Lets kernels be launched with up to `bytes` of dynamic shared memory on the current device: the most that any call asks for, since
// the limit belongs to the kernel and a smaller call's would take it from a larger one on another thread.
template <typename... Kernels>
int allow_smem(OncePerDevice& once, size_t bytes, Kernels... kernels) {
  return once(current_device(), [&]() -> int {
    for (const void* k : {reinterpret_cast<const void*>(kernels)...}) FLOP_CUDA(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return FLOP_OK;
  });
}

inline int num_sms() {
  static int cached[kMaxDevices] = {};
  const int dev = current_device();
  if (dev >= 0 && cached[dev]) return cached[dev];
  int n = 0;
  if (dev < 0 || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    return 148;   // B200; used only for planning when no device is visible
  }
  cached[dev] = n;
  return n;
}

// Host-side count of kernels launched by this library.
inline unsigned long long g_launches = 0;
inline void count_launch(int n = 1) { g_launches += (unsigned long long)n; }

// ------------------------------------------------------------------ bump allocator over ws
struct Arena {
  unsigned char* base;
  size_t size, used;
  void* take(size_t bytes) {
    const size_t off = align_up(used, 256);
    used = off + bytes;
    return base ? base + off : nullptr;
  }
};

inline bool check_mat(const void* p, int64_t ld, int64_t cols) { return p != nullptr && ld >= cols; }
inline bool bf16_ok(const void* p, int64_t ld) { return aligned16(p) && (ld % 8) == 0; }

inline int check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return FLOP_OK;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || ws_bytes < need) return FLOP_ERR_WORKSPACE;
  return FLOP_OK;
}

}  // namespace flop
