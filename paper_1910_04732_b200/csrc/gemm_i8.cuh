// 8-bit tensor-core GEMM for sm_100a: D[M,N] = sum_k A[m,k] B[n,k], both operands K-major 8-bit integers, exact 32-bit sums in tensor
// memory (tcgen05.mma kind::i8), scaled back to Y = D * a_scale[m] * b_scale[n] in the epilogue.
//
// Roles, barriers, pair protocol and bounded waits are those of gemm_tc.cuh / gemm_tc2.cuh: a 128-byte swizzle row holds 128 values of K
// instead of 64, an instruction takes 32 of them instead of 16, so a k-block moves the bytes of a bf16 one, takes its cycles, and does twice the work.
// Every CTA (or CTA pair) is persistent and walks the tiles in turn, all N tiles of a row block next to one another; two accumulators
// overlap the epilogue of a tile with the main loop of the next.
// Epilogue: a thread holds a row, so its token's scale is one register; the channels' scales of its columns are in shared memory before
// the accumulator is there.  bf16 leaves through a swizzled 32 x 64 staging tile and a TMA store (which clips the edges), 32-bit results through
// the same tile as coalesced stores.
//
// Bound: tensor cores, then power.  16384 x 6144 x 2048 bf16 142 us, 2.91 POP/s (87 % of twice the measured bf16 product), until the power cap
// takes hold: 160 us at 1490 MHz when calls follow one another for milliseconds.  8192 x 8192 x 8192 425-434 us, 2.5-2.6 POP/s under the cap.  Short K is
// bound by the epilogue (4096 x 4096: 11.3 us for K = 128, 13.5 for 358, 17.0 for 1024), so both 64-column halves are fetched at once and its loops
// are unrolled (a loop over them: 7 % slower; fp32 results of CTA pairs spill 40 bytes a thread that way).
#pragma once
#include "gemm_tc2.cuh"
#include "quantized.cuh"

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

constexpr uint32_t kWarpScales = 128 * 4;         // bytes: the scales of the (up to 128) columns that an epilogue warp takes of a tile
constexpr uint32_t kScalesTotal = tc::kEpiWarps * kWarpScales;
constexpr uint32_t kStage2 = 2 * tc::kStoreBufTotal;                   // two staging tiles per epilogue warp

__device__ __forceinline__ void ld_shared_v4(uint32_t addr, float (&v)[4]) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
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
// Warp h of a row quarter takes the 64-column groups h and h + 2 of a tile: their scales, before the accumulator is waited for.
__device__ __forceinline__ void fetch_scales(const GemmParams& p, uint32_t scales, int n_base, int n_end, int h, int lane) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int n = n_base + 64 * (h + 2 * i) + 2 * lane;
    const float a = n < n_end ? __ldg(p.b_scale + n) : 0.f, b = n + 1 < n_end ? __ldg(p.b_scale + n + 1) : 0.f;
    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(scales + 256u * i + 8u * lane), "f"(a), "f"(b) : "memory");
  }
  __syncwarp();
}
// v[0..3] scaled: (float(sum) * sa) * scale
__device__ __forceinline__ void scale4(const uint32_t* v, uint64_t sa2, uint32_t scales, float (&out)[4]) {
  float sc[4];
  ld_shared_v4(scales, sc);
  const float2 x = unpack2(mul2(mul2(pack2((float)(int)v[0], (float)(int)v[1]), sa2), pack2(sc[0], sc[1])));
  const float2 y = unpack2(mul2(mul2(pack2((float)(int)v[2], (float)(int)v[3]), sa2), pack2(sc[2], sc[3])));
  out[0] = x.x; out[1] = x.y; out[2] = y.x; out[3] = y.y;
}

// One accumulator tile through one epilogue warp (see tc::run_epilogue): q = warp & 3 fixes its 32 rows, h which 64-column groups it takes.  Both
// groups are fetched from tensor memory before anything is converted, so the accumulator is handed back at once; each has a staging
// tile of its own, so neither waits for the other's store.
template <int OUT, bool PAIR>
__device__ __forceinline__ void epilogue(const GemmParams& p, uint32_t buf, uint32_t scales, uint32_t t_acc, int row0, int n_base, int warp, int lane, uint32_t release_bar) {
  using namespace tc;
  const int q = warp & 3, h = (warp - 2) >> 2, row_base = row0 + q * 32, row = row_base + lane;
  const uint32_t t_row = t_acc + ((uint32_t)(q * 32) << 16);
  const int n_end = min(n_base + p.bn, p.N), nchunks = (n_end - n_base + 31) >> 5;
  const float sa = OUT != OUT_S32 && row < p.M ? __ldg(p.a_scale + row) : 0.f;
  const uint64_t sa2 = pack2(sa, sa);
  uint32_t v[4][32];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = 2 * (h + 2 * (i >> 1)) + (i & 1);
    if (c < nchunks) tmem_ld32(t_row + (uint32_t)(c * 32), v[i]);
  }
  tmem_ld_wait();
  tcgen05_fence_before();
  __syncwarp();
  if (lane == 0) {
    if (PAIR) mbar_arrive_remote(release_bar);
    else mbar_arrive(release_bar);
    if (OUT == OUT_BF16) tma_store_wait_read();        // the stores of the tile before have left the staging tiles
  }
  __syncwarp();
  if (OUT == OUT_BF16) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int c0 = 2 * (h + 2 * g), n0 = n_base + c0 * 32;
      if (c0 >= nchunks) break;
      // a store of the engine that ends inside a 16-byte piece writes the piece whole: the columns behind N are the caller's
      const bool edge = n0 + 64 > p.N && (p.N & 7);
      const uint32_t tile = buf + (uint32_t)g * kStoreBufBytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i == 4 && c0 + 1 >= nchunks) break;
        float f[8];
        scale4(v[2 * g + (i >> 2)] + 8 * (i & 3), sa2, scales + 256u * g + 32u * i, *reinterpret_cast<float(*)[4]>(f));
        scale4(v[2 * g + (i >> 2)] + 8 * (i & 3) + 4, sa2, scales + 256u * g + 32u * i + 16u, *reinterpret_cast<float(*)[4]>(f + 4));
        uint32_t pk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
          pk[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
        if (!edge) {
          st_shared_v4(tile + (uint32_t)lane * 128u + (uint32_t)((i ^ (lane & 7)) << 4), pk[0], pk[1], pk[2], pk[3]);
        } else if (row < p.M) {
          const int n = n0 + 8 * i;
          __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)row * p.ldo + n;
          if (n + 8 <= p.N) *reinterpret_cast<uint4*>(o) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          else
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (n + e < p.N) o[e] = reinterpret_cast<const __nv_bfloat16*>(pk)[e];
        }
      }
      if (edge) continue;
      fence_async_smem();
      __syncwarp();
      if (lane == 0 && row_base < p.M) tma_store_2d(&p.tout, n0, row_base, tile);      // never start a store outside the tensor
    }
    return;
  }
  // 32-bit results: a chunk at a time through the staging tiles in turn, then four rows of 128 bytes per instruction
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = 2 * (h + 2 * (i >> 1)) + (i & 1), n0 = n_base + c * 32;
    if (c >= nchunks) break;
    const uint32_t tile = buf + (uint32_t)(i & 1) * kStoreBufBytes;
    if (i >= 2) __syncwarp();                          // the chunk before last has been read out of this tile
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (OUT == OUT_F32) {
        float f[4];
        scale4(v[i] + 4 * j, sa2, scales + 128u * i + 16u * j, f);
        st_shared_v4(tile + (uint32_t)lane * 128u + (uint32_t)((j ^ (lane & 7)) << 4), __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
      } else {
        st_shared_v4(tile + (uint32_t)lane * 128u + (uint32_t)((j ^ (lane & 7)) << 4), v[i][4 * j], v[i][4 * j + 1], v[i][4 * j + 2], v[i][4 * j + 3]);
      }
    }
    __syncwarp();
    uint32_t* out = reinterpret_cast<uint32_t*>(p.out) + (int64_t)row_base * p.ldo + n0;
    if (p.vec && n0 + 32 <= n_end) {
      const int r0 = lane >> 3, c4 = lane & 7;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = r0 + 4 * j;
        uint4 w;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                     : "r"(tile + (uint32_t)r * 128u + (uint32_t)((c4 ^ (r & 7)) << 4)) : "memory");
        if (row_base + r < p.M) *reinterpret_cast<uint4*>(out + (int64_t)r * p.ldo + 4 * c4) = w;
      }
    } else {
      const int rows = min(32, p.M - row_base);
      for (int r = 0; r < rows; ++r) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(tile + (uint32_t)r * 128u + (uint32_t)(((lane >> 2) ^ (r & 7)) << 4) + 4u * (lane & 3)) : "memory");
        if (n0 + lane < n_end) out[(int64_t)r * p.ldo + lane] = w;
      }
    }
  }
  __syncwarp();
}

template <int OUT, bool PAIR>
__global__ void __launch_bounds__(tc::kThreads, 1)
gemm_kernel(const __grid_constant__ GemmParams p) {
  using namespace tc;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sbytes = PAIR ? stage_bytes2(p.bn) : stage_bytes(p.bn);
  const uint32_t store_base = smem_base + (uint32_t)p.stages * sbytes;
  const uint32_t scale_base = store_base + kStage2, bar_base = scale_base + kScalesTotal;
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
      const uint32_t scales = scale_base + (uint32_t)(warp - 2) * kWarpScales;
      if (OUT != OUT_S32) fetch_scales(p, scales, tn * p.bn, min(tn * p.bn + p.bn, p.N), (warp - 2) >> 2, lane);
      ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(acc), acc_phase, abort_flag));
      if (!ok) break;
      tcgen05_fence_after();
      epilogue<OUT, PAIR>(p, store_base + (uint32_t)(warp - 2) * 2 * kStoreBufBytes, scales, tmem_base + (uint32_t)acc * acc_stride(p.bn), tm * bm + (int)rank * BM, tn * p.bn,
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

// ---- first product of a compact pair, its rows quantised again before they leave the SM: Hq = 127 h / max |h| rounded, h = sum * col_scale, and
// h_scale = a_scale * max |h| / 127.  A row's maximum needs all of its columns: a cluster of one to four CTAs holds a 128-row block, each a slice of
// up to 256 columns in tensor memory, and they exchange the maxima of their slices through distributed shared memory.  That saves the trip of
// the 32-bit sums through memory and a launch that would be waited for.
//
// The maximum is that of the exact products.  A sum below 2^24 is exact in fp32, so x = fl(sum * scale) is its product rounded once, rounding
// keeps the order, and the largest product is among those with the largest x: the one with the largest rounding error, which an fma gives
// exactly.  Rows beyond that (longer sums, products outside 1e+-30) are compared in fp64.  Rounding as everywhere: in fp32 unless
// the quotient is within its error of a border.
constexpr int kRowqMaxSlice = 256, kRowqMaxCluster = 4;

struct RowqParams {
  CUtensorMap ta, tb;
  int M, N, num_kb, slice, stages, parts;         // N columns in `parts` slices
  const float *a_scale, *col_scale;
  int8_t* out; int64_t ldo; float* h_scale;
};
__host__ __device__ inline uint32_t rowq_stage_bytes(int slice) { return tc::kATileBytes + (uint32_t)slice * kBK; }
constexpr uint32_t kRowqFixed = 1024 + kRowqMaxSlice * 4 + kRowqMaxCluster * 2 * 128 * 8 + 384;

__device__ __noinline__ uint32_t round_sum(int sum, float scale, double exact, float inv) {
  const double x = (double)sum * (double)scale;
  const int q = exact < 1e30 && exact > 1e-30 ? round_border(x, exact, (int)floorf((float)sum * scale * inv)) : (int)rint(127.0 * x / exact);
  return (uint32_t)q & 255u;
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(taddr) : "memory");
  tc::tmem_ld_wait();
}
// A thread walks its columns eight at a time in loops that are not unrolled: it does so once or twice in its life, and code that runs once waits
// for its instructions (32 columns at a time, unrolled: 1.5 us per 32 columns).
__global__ void __launch_bounds__(tc::kThreads, 1)
gemm_rowq_kernel(const __grid_constant__ RowqParams p) {
  using namespace tc;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sbytes = rowq_stage_bytes(p.slice);
  const uint32_t scale_base = smem_base + (uint32_t)p.stages * sbytes, max_base = scale_base + kRowqMaxSlice * 4;
  const uint32_t bar_base = max_base + kRowqMaxCluster * 2 * 128 * 8;
  auto full_bar = [&](int s) { return bar_base + 8u * (uint32_t)s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (uint32_t)(kMaxStages + s); };
  const uint32_t tfull = bar_base + 8u * (uint32_t)(2 * kMaxStages);
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = blockIdx.x % p.parts, tm = blockIdx.x / p.parts;
  const int n_base = part * p.slice, n_end = min(n_base + p.slice, p.N);
  const bool work = n_base < p.N;                                         // (a last slice can be empty)
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < p.stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(tfull, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && lane == 0) { prefetch_tmap(&p.ta); prefetch_tmap(&p.tb); }
  if (warp == 1) tmem_alloc(smem_u32(&s_tmem_base), kRowqMaxSlice);
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  volatile int* abort_flag = &s_abort;
  pdl_wait();
  pdl_launch_dependents();
  cluster_sync_all();                                                     // every CTA is there before one stores to another

  if (warp == 0) {
    if (lane == 0 && work) {
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) break;
        const uint32_t sa = smem_base + (uint32_t)stage * sbytes;
        mbar_expect_tx(full_bar(stage), sbytes);
        tma_load_2d(sa, &p.ta, kb * kBK, tm * BM, full_bar(stage));
        tma_load_2d(sa + kATileBytes, &p.tb, kb * kBK, n_base, full_bar(stage));
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
      }
      if (*abort_flag) {
        const long long t0 = clock64();                                   // leaving early: let the copies already issued land
        while (clock64() - t0 < 2000000LL) {}
      }
    }
    __syncwarp();
    cluster_sync_all();
  } else if (warp == 1) {
    if (lane == 0 && work) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t idesc = instr_desc_s8(BM, p.slice);
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if (!mbar_wait(full_bar(stage), phase, abort_flag)) { ok = false; break; }
        tcgen05_fence_after();
        const uint32_t sa = smem_base + (uint32_t)stage * sbytes, sb = sa + kATileBytes;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma_s8<false>(tmem_base, smem_desc(sa + k * 32, false), smem_desc(sb + k * 32, false), idesc, (kb > 0 || k > 0) ? 1u : 0u);
        umma_commit(empty_bar(stage));
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
      }
      if (ok) umma_commit(tfull);
    }
    __syncwarp();
    cluster_sync_all();
  } else {
    const int q = warp & 3, h = (warp - 2) >> 2, r = q * 32 + lane, row = tm * BM + r;
    const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16);
    const int nchunks = work ? (n_end - n_base + 31) >> 5 : 0;
    for (int i = threadIdx.x - 64; i < kRowqMaxSlice; i += 32 * kEpiWarps) {
      const float s = n_base + i < n_end ? __ldg(p.col_scale + n_base + i) : 0.f;
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(scale_base + 4u * (uint32_t)i), "f"(s) : "memory");
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const bool ok = __all_sync(0xffffffffu, !work || mbar_wait(tfull, 0u, abort_flag));
    tcgen05_fence_after();
    // the largest product of this thread's columns: rounded, and its rounding error
    float top = 0.f, rest = 0.f;
    int longest = 0;
    // this thread's: 16 h .. 16 h + 15 of every 32, up to the slice's end (a multiple of 16): what lies in tensor memory behind it is an older kernel's
    const int cols_here = ok ? min(nchunks * 32, p.slice) : 0;
    auto next_cols = [](int n) { return n + ((n & 8) ? 24 : 8); };
#pragma unroll 1
    for (int n = 16 * h; n < cols_here; n = next_cols(n)) {
      uint32_t v[8];
      float sc[8], x[8], here = 0.f;
      tmem_ld8(t_row + (uint32_t)n, v);
      ld_shared_v4(scale_base + 4u * (uint32_t)n, *reinterpret_cast<float(*)[4]>(sc));
      ld_shared_v4(scale_base + 4u * (uint32_t)n + 16u, *reinterpret_cast<float(*)[4]>(sc + 4));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        longest = max(longest, abs((int)v[e]));
        x[e] = fabsf((float)(int)v[e] * sc[e]);
        here = __uint_as_float(max(__float_as_uint(here), __float_as_uint(x[e])));      // (a NaN is the largest)
      }
      if (__float_as_uint(here) >= __float_as_uint(top)) {                // (bits again: a NaN is not replaced)
        if (!(here == top)) rest = -INFINITY;
        top = here;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (x[e] == top) rest = fmaxf(rest, fmaf(fabsf((float)(int)v[e]), fabsf(sc[e]), -x[e]));
      }
    }
    double best = (double)top + (double)rest;
    // not decided by that: sums beyond 24 bits, products that fp32 does not hold
    const bool far = longest > (1 << 24) || (longest > 0 && !(top < 1e30f && top > 1e-30f));
    if (__any_sync(0xffffffffu, far)) {
      double b = 0.0;
#pragma unroll 1
      for (int n = 16 * h; n < cols_here; n = next_cols(n)) {
        uint32_t v[8];
        tmem_ld8(t_row + (uint32_t)n, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float sc;
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(sc) : "r"(scale_base + 4u * (uint32_t)(n + e)) : "memory");
          const double x = fabs((double)(int)v[e] * (double)sc);
          b = x < (double)INFINITY ? fmax(b, x) : (double)INFINITY;
        }
      }
      if (far) best = b;
    }
    if (!(best < (double)INFINITY)) best = (double)INFINITY;              // a channel without a scale: so is the row, and fmax below would drop a NaN
    // every CTA's maxima to every CTA, then the row's
    {
      const uint32_t at = max_base + (uint32_t)(((part * 2 + h) * 128 + r) * 8);
      for (int i = 0; i < p.parts; ++i)
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(map_to_cta(at, (uint32_t)i)), "d"(best) : "memory");
    }
    __syncwarp();
    cluster_sync_all();
    double exact = 0.0;
    for (int i = 0; i < 2 * p.parts; ++i) {
      double x;
      asm volatile("ld.shared.f64 %0, [%1];" : "=d"(x) : "r"(max_base + (uint32_t)((i * 128 + r) * 8)) : "memory");
      exact = fmax(exact, x);
    }
    const bool finite = exact < (double)INFINITY, plain = exact < 1e30 && exact > 1e-30;
    if (ok && part == 0 && h == 0 && row < p.M) p.h_scale[row] = finite ? (float)((double)__ldg(p.a_scale + row) * (exact * (1.0 / 127.0))) : NAN;
    const float inv = plain ? 127.f / (float)exact : 0.f;
    const int cols = min((p.N + 15) & ~15, n_base + p.slice);             // whole 16-byte pieces, zeros behind N; the slice behind this one writes its own
    int8_t* out = p.out + (int64_t)row * p.ldo + n_base;
    uint2 half = make_uint2(0, 0);
#pragma unroll 1
    for (int n = 16 * h; n < cols_here; n = next_cols(n)) {
      uint32_t v[8], b[8], near = 0;
      float sc[8];
      tmem_ld8(t_row + (uint32_t)n, v);
      ld_shared_v4(scale_base + 4u * (uint32_t)n, *reinterpret_cast<float(*)[4]>(sc));
      ld_shared_v4(scale_base + 4u * (uint32_t)n + 16u, *reinterpret_cast<float(*)[4]>(sc + 4));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = (float)(int)v[e] * sc[e], s = fmaf(x, inv, kToInt), off = fmaf(x, inv, kToInt - s);
        b[e] = __float_as_uint(s);
        near |= fabsf(off) >= 0.5f - kBorderSums ? 1u << e : 0u;
      }
      if (!plain) near = finite && exact > 0.0 ? 255u : 0u;
#pragma unroll 1
      for (; near; near &= near - 1) {
        const int e = __ffs(near) - 1;
        int s = 0;
        float scale = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i == e) { s = (int)v[i]; scale = sc[i]; }
        const uint32_t q8 = round_sum(s, scale, exact, inv);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = i == e ? q8 : b[i];
      }
      const uint2 w = finite ? bytes8(b) : make_uint2(0, 0);
      if (!(n & 8)) half = w;
      else if (row < p.M && n_base + n - 8 < cols) *reinterpret_cast<uint4*>(out + n - 8) = make_uint4(half.x, half.y, w.x, w.y);
    }
  }
  tcgen05_fence_before();
  __syncthreads();
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_dealloc(tmem_base, kRowqMaxSlice);
  }
}

}  // namespace i8
}  // namespace flop
