// 8-bit tensor-core GEMM for sm_100a: D[M,N] = sum_k A[m,k] B[n,k], both operands K-major 8-bit integers, exact 32-bit sums in tensor
// memory (tcgen05.mma kind::i8), scaled back to Y = D * a_scale[m] * b_scale[n] in the epilogue.
//
// Roles, barriers, pair protocol and bounded waits are those of gemm_tc.cuh / gemm_tc2.cuh: a 128-byte swizzle row holds 128 values of K
// instead of 64, an instruction takes 32 of them instead of 16, so a k-block moves the bytes of a bf16 one, takes its cycles, and does twice the work.
// Every CTA (or CTA pair) is persistent and walks the tiles in turn, all N tiles of a row block next to one another; two accumulators
// overlap the epilogue of a tile with the main loop of the next.
// Epilogue: a thread holds a row, so its token's scale is one register; the channels' scales of a 32-column chunk come as broadcast
// 16-byte loads.  bf16 leaves through a swizzled 32 x 64 staging tile and a TMA store (which clips the edges), 32-bit results through
// the same tile as coalesced stores.
#pragma once
#include "gemm_tc2.cuh"

namespace flop {
namespace i8 {

constexpr int kBK = 128;                          // K per stage: one 128-byte swizzle row
enum { OUT_BF16 = 0, OUT_F32 = 1, OUT_S32 = 2 };

struct GemmParams {
  CUtensorMap ta, tb, tout;                       // tout: bf16 results only
  int M, N, num_kb, bn, tiles_m, tiles_n, stages;
  const float *a_scale, *b_scale;
  void* out; int64_t ldo; int vec;                // vec: rows of 32-bit results start on 16 bytes
};

__device__ __forceinline__ uint32_t instr_desc_s8(int m, int n) {      // s32 accumulators, s8 A and B, both K-major
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <bool PAIR>
__device__ __forceinline__ void umma_s8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

// the scales of 32 columns, 0 behind the last one (`vec`: b_scale + n0 is 16-byte aligned)
__device__ __forceinline__ void load_scales(const float* __restrict__ b_scale, int n0, int N, float (&sc)[32]) {
  if (n0 + 32 <= N && (reinterpret_cast<uintptr_t>(b_scale + n0) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(b_scale + n0) + i);
      sc[4 * i] = f.x; sc[4 * i + 1] = f.y; sc[4 * i + 2] = f.z; sc[4 * i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) sc[i] = n0 + i < N ? __ldg(b_scale + n0 + i) : 0.f;
  }
}

// One accumulator tile through one epilogue warp (see tc::run_epilogue): q = warp & 3 fixes its 32 rows, h its share of the 32-column chunks.
template <int OUT, bool PAIR>
__device__ __forceinline__ void epilogue(const GemmParams& p, uint32_t buf, uint32_t t_acc, int row0, int n_base, int warp, int lane, uint32_t release_bar) {
  using namespace tc;
  const int q = warp & 3, h = (warp - 2) >> 2, row_base = row0 + q * 32, row = row_base + lane;
  const uint32_t t_row = t_acc + ((uint32_t)(q * 32) << 16);
  const int n_end = min(n_base + p.bn, p.N), nchunks = (n_end - n_base + 31) >> 5, ngroups = (nchunks + 1) >> 1;
  const float sa = OUT != OUT_S32 && row < p.M ? __ldg(p.a_scale + row) : 0.f;
  auto release = [&] {
    tcgen05_fence_before();
    __syncwarp();
    if (lane == 0) {
      if (PAIR) mbar_arrive_remote(release_bar);
      else mbar_arrive(release_bar);
    }
  };
  bool released = false;
  if (OUT == OUT_BF16) {
    for (int g = h; g < ngroups; g += 2) {
      const int c0 = 2 * g;
      const bool two = c0 + 1 < nchunks;
      uint32_t v[2][32];
      tmem_ld32(t_row + (uint32_t)(c0 * 32), v[0]);
      if (two) tmem_ld32(t_row + (uint32_t)(c0 * 32 + 32), v[1]);
      tmem_ld_wait();
      if (g + 2 >= ngroups) { release(); released = true; }
      const int n0 = n_base + c0 * 32;
      // a store of the engine that ends inside a 16-byte piece writes the piece whole: the columns behind N are the caller's
      const bool edge = n0 + 64 > p.N && (p.N & 7);
      if (lane == 0) tma_store_wait_read();            // the previous block has left the staging tile
      __syncwarp();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half && !two) break;
        float sc[32];
        load_scales(p.b_scale, n0 + 32 * half, p.N, sc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t pk[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = 8 * i + 2 * j;
            const __nv_bfloat162 b = __floats2bfloat162_rn((float)(int)v[half][e] * sa * sc[e], (float)(int)v[half][e + 1] * sa * sc[e + 1]);
            pk[j] = *reinterpret_cast<const uint32_t*>(&b);
          }
          if (!edge) {
            st_shared_v4(buf + (uint32_t)lane * 128u + (uint32_t)(((4 * half + i) ^ (lane & 7)) << 4), pk[0], pk[1], pk[2], pk[3]);
          } else if (row < p.M) {
            const int n = n0 + 32 * half + 8 * i;
            __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)row * p.ldo + n;
            if (n + 8 <= p.N) *reinterpret_cast<uint4*>(o) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            else
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (n + e < p.N) o[e] = reinterpret_cast<const __nv_bfloat16*>(pk)[e];
          }
        }
      }
      if (edge) continue;
      fence_async_smem();
      __syncwarp();
      if (lane == 0 && row_base < p.M) tma_store_2d(&p.tout, n0, row_base, buf);      // never start a store outside the tensor
    }
    if (!released) release();
    return;
  }
  // 32-bit results: a chunk at a time through the staging tile, then four rows of 128 bytes per instruction
#pragma unroll 1
  for (int c = h; c < nchunks; c += 2) {
    uint32_t v[32];
    tmem_ld32(t_row + (uint32_t)(c * 32), v);
    tmem_ld_wait();
    if (c + 2 >= nchunks) { release(); released = true; }
    const int n0 = n_base + c * 32;
    if (OUT == OUT_F32) {
      float sc[32];
      load_scales(p.b_scale, n0, p.N, sc);
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = __float_as_uint((float)(int)v[i] * sa * sc[i]);
    }
    __syncwarp();                                      // the previous chunk has been read out of the staging tile
#pragma unroll
    for (int i = 0; i < 8; ++i)
      st_shared_v4(buf + (uint32_t)lane * 128u + (uint32_t)((i ^ (lane & 7)) << 4), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    __syncwarp();
    uint32_t* out = reinterpret_cast<uint32_t*>(p.out) + (int64_t)row_base * p.ldo + n0;
    if (p.vec && n0 + 32 <= n_end) {
      const int r0 = lane >> 3, c4 = lane & 7;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 4 * i;
        uint4 w;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                     : "r"(buf + (uint32_t)r * 128u + (uint32_t)((c4 ^ (r & 7)) << 4)) : "memory");
        if (row_base + r < p.M) *reinterpret_cast<uint4*>(out + (int64_t)r * p.ldo + 4 * c4) = w;
      }
    } else {
      const int rows = min(32, p.M - row_base);
      for (int r = 0; r < rows; ++r) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(buf + (uint32_t)r * 128u + (uint32_t)(((lane >> 2) ^ (r & 7)) << 4) + 4u * (lane & 3)) : "memory");
        if (n0 + lane < n_end) out[(int64_t)r * p.ldo + lane] = w;
      }
    }
  }
  if (!released) release();
}

template <int OUT, bool PAIR>
__global__ void __launch_bounds__(tc::kThreads, 1)
gemm_kernel(const __grid_constant__ GemmParams p) {
  using namespace tc;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sbytes = PAIR ? stage_bytes2(p.bn) : stage_bytes(p.bn);
  const uint32_t store_base = smem_base + (uint32_t)p.stages * sbytes;
  const uint32_t bar_base = store_base + kStoreBufTotal;
  auto full_bar = [&](int s) { return bar_base + 8u * (uint32_t)s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (uint32_t)(kMaxStages + s); };
  auto tfull_bar = [&](int a) { return bar_base + 8u * (uint32_t)(2 * kMaxStages + a); };
  auto tempty_bar = [&](int a) { return bar_base + 8u * (uint32_t)(2 * kMaxStages + 2 + a); };
  const uint32_t exit_bar = bar_base + 8u * (uint32_t)(2 * kMaxStages + 4);
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int items = p.tiles_m * p.tiles_n, bm = PAIR ? BM2 : BM;

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < p.stages; ++s) { mbar_init(full_bar(s), PAIR ? 2 : 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), (PAIR ? 2 : 1) * kEpiWarps); }
    mbar_init(exit_bar, 2);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && lane == 0) {
    prefetch_tmap(&p.ta); prefetch_tmap(&p.tb);
    if (OUT == OUT_BF16) prefetch_tmap(&p.tout);
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc2(smem_u32(&s_tmem_base), kTmemCols);
    else tmem_alloc(smem_u32(&s_tmem_base), kTmemCols);
  }
  tcgen05_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  tcgen05_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  volatile int* abort_flag = &s_abort;
  pdl_wait();
  pdl_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int half_n = PAIR ? p.bn >> 1 : p.bn;
      const uint32_t tx = kATileBytes + (uint32_t)half_n * kBK;
      for (int w = unit; w < items && ok; w += units) {
        const int tm = w / p.tiles_n, tn = w - tm * p.tiles_n;
        const int m_base = tm * bm + (int)rank * BM, n_base = tn * p.bn + (int)rank * half_n;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t sa = smem_base + (uint32_t)stage * sbytes, sb = sa + kATileBytes;
          if (PAIR) {
            const uint32_t fb = map_to_cta(full_bar(stage), 0);
            mbar_expect_tx_cluster(fb, tx);
            tma_load_2d_pair(sa, &p.ta, kb * kBK, m_base, fb);
            tma_load_2d_pair(sb, &p.tb, kb * kBK, n_base, fb);
          } else {
            mbar_expect_tx(full_bar(stage), tx);
            tma_load_2d(sa, &p.ta, kb * kBK, m_base, full_bar(stage));
            tma_load_2d(sb, &p.tb, kb * kBK, n_base, full_bar(stage));
          }
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok || *abort_flag) {
        const long long t0 = clock64();                // leaving early: let the copies already issued land
        while (clock64() - t0 < 2000000LL) {}
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer (the leader's)
    if (lane == 0 && rank == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      const uint32_t idesc = instr_desc_s8(bm, p.bn), stride = acc_stride(p.bn);
      for (int w = unit; w < items && ok; w += units) {
        if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag)) { ok = false; break; }
        tcgen05_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)acc * stride;
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!mbar_wait(full_bar(stage), phase, abort_flag)) { ok = false; break; }
          tcgen05_fence_after();
          const uint32_t sa = smem_base + (uint32_t)stage * sbytes, sb = sa + kATileBytes;
#pragma unroll
          for (int k = 0; k < 4; ++k)                  // 32 values of K, 32 bytes, per instruction
            umma_s8<PAIR>(d_tmem, smem_desc(sa + k * 32, false), smem_desc(sb + k * 32, false), idesc, (kb > 0 || k > 0) ? 1u : 0u);
          if (PAIR) umma2_commit_mc(empty_bar(stage), 3);
          else umma_commit(empty_bar(stage));
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (PAIR) umma2_commit_mc(tfull_bar(acc), 3);
        else umma_commit(tfull_bar(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue warps
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int w = unit; w < items && ok; w += units) {
      const int tm = w / p.tiles_n, tn = w - tm * p.tiles_n;
      ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(acc), acc_phase, abort_flag));
      if (!ok) break;
      tcgen05_fence_after();
      epilogue<OUT, PAIR>(p, store_base + (uint32_t)(warp - 2) * kStoreBufBytes, tmem_base + (uint32_t)acc * acc_stride(p.bn), tm * bm + (int)rank * BM, tn * p.bn,
                          warp, lane, PAIR ? map_to_cta(tempty_bar(acc), 0) : tempty_bar(acc));
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
    if (OUT == OUT_BF16 && lane == 0) tma_store_wait_all();
  }
  // ---------------------------------------------------------------- teardown
  tcgen05_fence_before();
  __syncthreads();
  if (PAIR) {
    if (threadIdx.x == 0) {
      mbar_arrive_cluster(map_to_cta(exit_bar, 0));
      mbar_arrive_cluster(map_to_cta(exit_bar, 1));
      const long long t0 = clock64();
      while (!mbar_try_wait_cluster_acq(exit_bar, 0)) {
        if (clock64() - t0 > kWaitCycles) { report_timeout(); break; }
      }
    }
    __syncthreads();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    if (PAIR) tmem_dealloc2(tmem_base, kTmemCols);
    else tmem_dealloc(tmem_base, kTmemCols);
  }
}

}  // namespace i8
}  // namespace flop
