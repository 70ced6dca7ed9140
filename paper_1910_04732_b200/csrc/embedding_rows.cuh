// Embedding lookup with a scale, Y[t] = scale E[ids[t]], and the table's gradient, dE[v] = scale sum over {t: ids[t] = v} of dY[t].
// Words outside the table are padding: a row of zeros, no gradient.
//
// The gradient sorts the tokens by word (stably: a word's tokens stay in the order of the batch) and adds up runs of equal words.  Sums are
// fp32; how a word's tokens are grouped depends on where its run meets the borders of chunks, or on how many there are (few_kernel), so that the same call
// gives the same bits.  Every row is written once, by one thread for each column.
//   sort_kernel   : one thread-block cluster sorts (word, token) pairs, least significant digit first; the blocks behind it clear dE
//                   meanwhile, because most rows of a large table stay empty.  Long batches are sorted by two launches a digit (sort_count_kernel,
//                   sort_move_kernel) on as many blocks as they fill
//   runs_kernel   : the sorted tokens in chunks of equal length, whatever the words: a word that fills half of a batch is
//                   as well spread over the machine as a batch of rare ones.  A run that lies within a chunk is written to dE; what a chunk holds of
//                   a run that crosses its border goes to the workspace
//   joints_kernel : adds up the parts of the runs that cross borders, in order
//   few_kernel    : few tokens need none of this: a warp for each token looks through all words, and the first of equal ones adds up
#pragma once
#include <cooperative_groups.h>

#include "rows8.cuh"

namespace flop {
namespace emb {

// ---------------------------------------------------------------- lookup
struct LookupArgs {
  const int32_t* ids; int64_t T;
  const void* E; int64_t lde; int64_t V;
  void* Y; int64_t ldy;
  float scale;
  int d, vec;
};

// LANES threads share a row of Y, NG units each (blockIdx.y: segments of LANES * NG units); a block takes RB rows of each set of threads, first their words, then all their
// units, then stores.  (A ring of rows copied ahead, which carries the other operators here, is slower: a row's address waits for its word.  Units dealt out
// over all rows without regard to where rows end cost 100 instructions each: 16384 x 2048 bf16 of 205 rows 16.3 us.)
template <typename T, int LANES, int NG, int RB>
__global__ void __launch_bounds__(256)
lookup_kernel(const LookupArgs a) {
  constexpr int ROWS = 256 / LANES, E = kUnit<T>, H = kPairs<T>;
  pdl_wait();
  pdl_launch_dependents();
  const int k = (threadIdx.x % LANES + blockIdx.y * (LANES * NG)) * E;
  const int64_t t0 = (int64_t)blockIdx.x * (ROWS * RB) + threadIdx.x / LANES;
  const uint64_t scale = pack2(a.scale, a.scale);
  int id[RB];
#pragma unroll
  for (int q = 0; q < RB; ++q) id[q] = t0 + q * ROWS < a.T ? a.ids[t0 + q * ROWS] : -1;
  uint4 x[RB][NG];
#pragma unroll
  for (int q = 0; q < RB; ++q) {
    const bool word = id[q] >= 0 && id[q] < a.V;
    const T* row = (const T*)a.E + (int64_t)(word ? id[q] : 0) * a.lde + k;
#pragma unroll
    for (int i = 0; i < NG; ++i) x[q][i] = load_unit(row + i * LANES * E, word ? a.d - k - i * LANES * E : 0, a.vec, id[q] + 1 < a.V);
  }
#pragma unroll
  for (int q = 0; q < RB; ++q) {
    if (t0 + q * ROWS >= a.T) break;
    const bool word = id[q] >= 0 && id[q] < a.V;         // zeros for padding, also where the scale is not finite
    T* row = (T*)a.Y + (t0 + q * ROWS) * a.ldy + k;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      uint64_t v[H];
      unpack_unit<T>(x[q][i], v);
#pragma unroll
      for (int j = 0; j < H; ++j) v[j] = word ? mul2(v[j], scale) : 0;
      const int n = a.d - k - i * LANES * E;
      if (n > 0) store_unit(row + i * LANES * E, pack_unit<T>(v), n, a.vec);
    }
  }
}

// ---------------------------------------------------------------- rows of zeros
struct ClearArgs { unsigned char* p; int64_t rows, row_bytes, pitch; int vec; };   // vec: rows start on 16 bytes; else they are fp32

// The last bytes of a row, an even number below 16.
__device__ __forceinline__ void clear_tail(unsigned char* at, int64_t left) {
  if (left & 8) { *reinterpret_cast<uint2*>(at) = make_uint2(0, 0); at += 8; }
  if (left & 4) { *reinterpret_cast<uint32_t*>(at) = 0; at += 4; }
  if (left & 2) *reinterpret_cast<uint16_t*>(at) = 0;
}
// Piece i of a row: 16 bytes, or what is left of them at its end; a value where rows do not start on 16 bytes.
__device__ __forceinline__ void clear_piece(unsigned char* row, int64_t i, const ClearArgs& a) {
  const int64_t left = a.row_bytes - i * 16;
  if (!a.vec) *reinterpret_cast<uint32_t*>(row + i * 4) = 0;
  else if (left >= 16) *reinterpret_cast<uint4*>(row + i * 16) = make_uint4(0, 0, 0, 0);
  else clear_tail(row + i * 16, left);
}
// Rows [0, rows) from p on but those that `skip` names, by `step` threads of which this is the first-th: a warp for a row, or a thread for a piece of a short one.
template <typename Skip>
__device__ __forceinline__ void clear_rows(unsigned char* p, int64_t rows, const ClearArgs& a, int64_t first, int64_t step, Skip&& skip) {
  const int64_t pieces = a.vec ? (a.row_bytes + 15) / 16 : a.row_bytes / 4;
  if (pieces >= 32) {
    for (int64_t r = first / 32; r < rows; r += step / 32) {
      if (skip(r)) continue;
#pragma unroll 4
      for (int64_t i = threadIdx.x & 31; i < pieces; i += 32) clear_piece(p + r * a.pitch, i, a);
    }
    return;
  }
  const int64_t total = rows * pieces, step_rows = step / pieces, step_pieces = step - step_rows * pieces;
  int64_t row = first / pieces, piece = first - row * pieces;
  for (int64_t i = first; i < total; i += step) {
    if (!skip(row)) clear_piece(p + row * a.pitch, piece, a);
    row += step_rows;
    piece += step_pieces;
    if (piece >= pieces) { piece -= pieces; ++row; }
  }
}
// All rows, by `blocks` blocks of which this is the block-th.  Rows without a gap are one run of bytes, in tiles of four pieces a thread.
// (Writing alone, the memory takes 5.9 TB/s of such tiles, and 4.2 of tiles of a megabyte.)
__device__ __forceinline__ void clear_all(const ClearArgs& a, int64_t block, int64_t blocks) {
  const int threads = blockDim.x;
  if (a.pitch == a.row_bytes) {
    const int64_t bytes = a.rows * a.row_bytes, head = min(bytes, (int64_t)(-reinterpret_cast<uintptr_t>(a.p) & 15)), pieces = (bytes - head) / 16;
    uint4* p = reinterpret_cast<uint4*>(a.p + head);
    for (int64_t t = block * threads * 4; t < pieces; t += blocks * threads * 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t i = t + u * threads + threadIdx.x;
        if (i < pieces) p[i] = make_uint4(0, 0, 0, 0);
      }
    }
    if (block == 0 && threadIdx.x == 0) {
      for (int64_t i = 0; i < head; i += 2) *reinterpret_cast<uint16_t*>(a.p + i) = 0;
      clear_tail(a.p + head + pieces * 16, (bytes - head) & 15);
    }
  } else {
    clear_rows(a.p, a.rows, a, block * threads + threadIdx.x, blocks * threads, [](int64_t) { return false; });
  }
}

// ---------------------------------------------------------------- sort
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kMaxDigitBits = 9;
constexpr int kSortHeld = 4;        // pairs of a thread in sort_kernel
constexpr int kSortBlock = kSortThreads * kSortHeld, kSortBlocks = 128;      // pairs of a block, blocks of a long batch at most

struct SortArgs {
  const int32_t* ids; int64_t T;
  uint32_t V;
  int passes, bits;                 // digits of a word, bits of a digit
  uint2* order[2];                  // (word, token) pairs, written in turn; the last pass writes order[0]
  int blocks;                       // blocks that sort
  uint32_t* counts;                 // long batches: [blocks][bins]
  ClearArgs clear;                  // what the other blocks clear (rows 0: nothing)
  __device__ __forceinline__ const uint2* from(int pass) const { return (passes - pass) & 1 ? order[1] : order[0]; }
  __device__ __forceinline__ uint2* to(int pass) const { return (passes - pass) & 1 ? order[0] : order[1]; }
  __device__ __forceinline__ uint2 pair(int pass, int64_t i) const {
    if (pass) return from(pass)[i];
    const int32_t id = ids[i];
    return make_uint2(min((uint32_t)id, V), (uint32_t)i);           // padding sorts behind every word
  }
};
// A counter and a set of lanes for every warp and digit, then the block's sums and where its pairs of a digit begin.
inline size_t sort_smem(int bits) { return (2 * (size_t)kSortWarps + 2) * (1u << bits) * 4; }
struct SortShared {
  uint32_t *mine, *lanes, *total, *base;
  int bins;
  __device__ __forceinline__ SortShared(uint32_t* sm, int bits) : bins(1 << bits) {
    mine = sm + (threadIdx.x >> 5) * bins;
    lanes = mine + kSortWarps * bins;
    total = sm + 2 * kSortWarps * bins;
    base = total + bins;
  }
  __device__ __forceinline__ void clear() const {
    for (int b = threadIdx.x & 31; b < bins; b += 32) mine[b] = lanes[b] = 0;
    __syncwarp();
  }
  // Pairs of the same digit before this lane's in the warp's run so far; the run grows by the 32 pairs.  Equal digits find one another in shared memory: a
  // ballot for each bit takes 1500 cycles with all warps of an SM at it, this 500.
  __device__ __forceinline__ uint32_t rank(uint32_t digit, bool on) const {
    const int lane = threadIdx.x & 31;
    if (on) atomicOr(lanes + digit, 1u << lane);
    __syncwarp();
    const uint32_t same = on ? lanes[digit] : 0, at = on ? mine[digit] : 0;
    __syncwarp();
    if (on && (same >> lane) == 1u) {                    // the highest lane of each digit
      mine[digit] = at + __popc(same);
      lanes[digit] = 0;
    }
    __syncwarp();
    return at + __popc(same & ((1u << lane) - 1));
  }
};
// Behind the last pair there are a few that are no words, so that whoever reads the order needs no bounds.
constexpr int kBehind = 16;
constexpr uint32_t kNoWord = 0xFFFFFFFFu;                // words are below 2^31
__device__ __forceinline__ void end_order(const SortArgs& a, int block) {
  if (block == 0 && threadIdx.x < kBehind) a.order[0][a.T + threadIdx.x] = make_uint2(kNoWord, 0);
}
// Pairs [lo, hi) of this warp.
__device__ __forceinline__ void warp_run(int64_t T, int block, int blocks, int64_t& lo, int64_t& hi) {
  const int64_t warps = (int64_t)blocks * kSortWarps, per = ((T + warps * 32 - 1) / (warps * 32)) * 32;
  lo = min(T, ((int64_t)block * kSortWarps + (threadIdx.x >> 5)) * per);
  hi = min(T, lo + per);
}

// The warps' counts of each digit become the number of pairs before the warp's; `total` gets the sums.  A thread takes a digit, or half the warps of one where there are
// twice as many threads.
__device__ __forceinline__ void scan_warps(uint32_t* sm, const SortShared& s) {
  __shared__ uint32_t half[kSortThreads / 2];
  constexpr int HALF = kSortWarps / 2;
  const int digit = threadIdx.x & (s.bins - 1), part = threadIdx.x / s.bins;
  const bool split = 2 * s.bins <= kSortThreads, on = part < (split ? 2 : 1);
  uint32_t* p = sm + digit + (split && part ? HALF * s.bins : 0);
  uint32_t v[HALF], sum = 0;
  if (on) {
#pragma unroll
    for (int h = 0; h < HALF; ++h) sum += v[h] = p[h * s.bins];
  }
  if (split && on && part == 0) half[digit] = sum;
  __syncthreads();
  if (on) {
    uint32_t before = split && part ? half[digit] : 0;
#pragma unroll
    for (int h = 0; h < HALF; ++h) {
      p[h * s.bins] = before;
      before += v[h];
    }
    if (!split) {
#pragma unroll
      for (int h = 0; h < HALF; ++h) v[h] = p[(HALF + h) * s.bins];
#pragma unroll
      for (int h = 0; h < HALF; ++h) {
        p[(HALF + h) * s.bins] = before;
        before += v[h];
      }
    }
    if (!split || part) s.total[digit] = before;
  }
}
// base of digit b = threadIdx.x: pairs of lower digits anywhere, and of this digit in blocks before (`ahead`).
__device__ __forceinline__ void place_digits(const SortShared& s, uint32_t all, uint32_t ahead) {
  __shared__ uint32_t sums[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (s.bins + 31) / 32;
  uint32_t inc = all;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t n = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += n;
  }
  if (warp < warps && lane == 31) sums[warp] = inc;
  __syncthreads();
  if ((int)threadIdx.x < s.bins) {
    uint32_t before = 0;
    for (int w = 0; w < warp; ++w) before += sums[w];
    s.base[threadIdx.x] = before + inc - all + ahead;
  }
  __syncthreads();
}

// A pass of a cluster of C blocks of 16 warps: warp w of block c owns the (c 16 + w)-th run of consecutive pairs, 128 at most.  It counts its digits;
// the block turns the counts into positions (over its warps in shared memory, over the blocks in distributed shared memory); the warp
// then moves every pair behind the ones of the same digit before it.  Within a group of 32 the order among equal digits is that of the lanes.
__global__ void __launch_bounds__(kSortThreads)
sort_kernel(const SortArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  if ((int)blockIdx.x >= a.blocks) {
    clear_all(a.clear, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    return;
  }
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ uint32_t sm[];
  const SortShared s(sm, a.bits);
  const int lane = threadIdx.x & 31, rank = (int)cluster.block_rank();
  int64_t lo, hi;
  warp_run(a.T, rank, a.blocks, lo, hi);
  end_order(a, rank);
  for (int pass = 0; pass < a.passes; ++pass) {
    uint2 held[kSortHeld];
    uint32_t before[kSortHeld], digit[kSortHeld];        // pairs of the same digit before it in the warp's run
#pragma unroll
    for (int h = 0; h < kSortHeld; ++h) held[h] = lo + h * 32 + lane < hi ? a.pair(pass, lo + h * 32 + lane) : make_uint2(0, 0);
    s.clear();
#pragma unroll
    for (int h = 0; h < kSortHeld; ++h) {
      digit[h] = (held[h].x >> (pass * a.bits)) & (s.bins - 1);
      before[h] = s.rank(digit[h], lo + h * 32 + lane < hi);
    }
    __syncthreads();
    scan_warps(sm, s);
    cluster.sync();
    uint32_t ahead = 0, all = 0;
    if ((int)threadIdx.x < s.bins) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {                      // all eight in flight, whether there are so many blocks or not
        const uint32_t v = *cluster.map_shared_rank(s.total + threadIdx.x, min(c, a.blocks - 1));
        if (c < a.blocks) all += v;
        if (c < rank) ahead += v;
      }
    }
    const bool more = pass + 1 < a.passes;
    if (!more) cluster.barrier_arrive();                 // the last look at the other blocks' memory
    place_digits(s, all, ahead);
    uint2* to = a.to(pass);
#pragma unroll
    for (int h = 0; h < kSortHeld; ++h)
      if (lo + h * 32 + lane < hi) to[s.base[digit[h]] + s.mine[digit[h]] + before[h]] = held[h];
    if (more) cluster.sync();                            // the pairs are in place and `total` has been read
    else cluster.barrier_wait();
  }
}

// A pass over a long batch, first launch: the digits of each block's run of pairs are counted.
__device__ __forceinline__ void count_run(const SortArgs& a, const SortShared& s, int pass, int64_t lo, int64_t hi) {
  const int lane = threadIdx.x & 31;
  s.clear();
  for (int64_t i = lo; i < hi; i += 64) {
    uint32_t digit[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) digit[h] = i + h * 32 + lane < hi ? (a.pair(pass, i + h * 32 + lane).x >> (pass * a.bits)) & (s.bins - 1) : (uint32_t)s.bins;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (digit[h] < (uint32_t)s.bins) atomicAdd(s.mine + digit[h], 1u);         // a count, whatever the order
  }
  __syncthreads();
}
__global__ void __launch_bounds__(kSortThreads)
sort_count_kernel(const SortArgs a, int pass) {
  pdl_wait();
  pdl_launch_dependents();
  if ((int)blockIdx.x >= a.blocks) {
    clear_all(a.clear, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    return;
  }
  extern __shared__ uint32_t sm[];
  const SortShared s(sm, a.bits);
  int64_t lo, hi;
  warp_run(a.T, blockIdx.x, a.blocks, lo, hi);
  count_run(a, s, pass, lo, hi);
  for (int b = threadIdx.x; b < s.bins; b += kSortThreads) {
    uint32_t n = 0;
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) n += sm[w * s.bins + b];
    a.counts[(int64_t)blockIdx.x * s.bins + b] = n;
  }
}
// Second launch: every block adds up the counts of all blocks and of those before it, and moves its pairs.
__global__ void __launch_bounds__(kSortThreads)
sort_move_kernel(const SortArgs a, int pass) {
  pdl_wait();
  pdl_launch_dependents();
  extern __shared__ uint32_t sm[];
  const SortShared s(sm, a.bits);
  const int lane = threadIdx.x & 31;
  uint32_t ahead = 0, all = 0;
  if ((int)threadIdx.x < s.bins) {
#pragma unroll 16
    for (int c = 0; c < a.blocks; ++c) {
      const uint32_t v = a.counts[(int64_t)c * s.bins + threadIdx.x];
      all += v;
      if (c < (int)blockIdx.x) ahead += v;
    }
  }
  int64_t lo, hi;
  warp_run(a.T, blockIdx.x, a.blocks, lo, hi);
  end_order(a, blockIdx.x);
  count_run(a, s, pass, lo, hi);
  scan_warps(sm, s);
  place_digits(s, all, ahead);
  uint2* to = a.to(pass);
  for (int64_t i = lo; i < hi; i += 64) {
    uint2 p[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) p[h] = i + h * 32 + lane < hi ? a.pair(pass, i + h * 32 + lane) : make_uint2(0, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool on = i + h * 32 + lane < hi;
      const uint32_t digit = (p[h].x >> (pass * a.bits)) & (s.bins - 1), at = s.rank(digit, on);
      if (on) to[s.base[digit] + at] = p[h];
    }
  }
}

// ---------------------------------------------------------------- runs of equal words
struct RunArgs {
  const uint2* order; int64_t T;
  const int32_t* ids;               // few_kernel
  uint32_t V;
  const void* dY; int64_t lddy;
  void* dE; int64_t ldde;
  float* part; int64_t part_ld;     // [chunks][2][part_ld]: a chunk's share of the run that comes from before it, of the one that goes on behind it
  int64_t chunks; int chunk;        // tokens of a chunk, a multiple of 4
  float scale;
  int d, slices;                    // slices of LPT * 8 columns
  int accumulate, vec, vec_out;
  ClearArgs clear; int clear_rows, token_blocks;       // few_kernel: rows that a block clears, blocks before those that do
};

// scale v (+)= into E columns of dE's row, n of which exist
template <typename TW, int E>
__device__ __forceinline__ void write_columns(const RunArgs& a, uint32_t word, int k, int n, const float (&v)[E]) {
  TW* p = (TW*)a.dE + (int64_t)word * a.ldde + k;
  constexpr int BYTES = E * (int)sizeof(TW);
  const bool whole = a.vec_out && n >= E;
  if constexpr (sizeof(TW) == 4) {
    // This thread alone writes here: the memory adds, and nothing waits for the old values (16384 fp32 rows of 1024 columns, 40000 words: 31.5 us; read, added and written 59.8).  It
    // takes subnormal values for zero.  What is no whole piece is read and written (by the memory, value by value: bf16 rows that start anywhere 90 us, 56 this way; and
    // few_kernel has 68 registers instead of 56 with a path for the ends of rows).
    if (a.accumulate && whole) {
#pragma unroll
      for (int j = 0; j < E; j += 4)
        atomicAdd(reinterpret_cast<float4*>(p + j), make_float4(a.scale * v[j], a.scale * v[j + 1], a.scale * v[j + 2], a.scale * v[j + 3]));
      return;
    }
  }
  TW out[E];
  if (a.accumulate) {
    if (whole) {
      if constexpr (BYTES == 8) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        memcpy(out, &q, 8);
      } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
          const uint4 q = reinterpret_cast<const uint4*>(p)[i];
          memcpy(reinterpret_cast<char*>(out) + 16 * i, &q, 16);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) out[j] = j < n ? p[j] : from_f32<TW>(0.f);
    }
  }
#pragma unroll
  for (int j = 0; j < E; ++j) out[j] = from_f32<TW>(a.accumulate ? __fadd_rn(__fmul_rn(a.scale, v[j]), to_f32(out[j])) : a.scale * v[j]);      // as the memory rounds
  if (whole) {
    if constexpr (BYTES == 8) {
      uint2 q;
      memcpy(&q, out, 8);
      *reinterpret_cast<uint2*>(p) = q;
    } else {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        uint4 q;
        memcpy(&q, reinterpret_cast<const char*>(out) + 16 * i, 16);
        reinterpret_cast<uint4*>(p)[i] = q;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (j < n) p[j] = out[j];
  }
}

// LPT lanes take a chunk's slice of LPT * 8 columns.  Their rows come through a ring of AHEAD steps of four, each thread copying and reading its own units:
// one batch of rows after another from memory would leave a warp waiting for most of its time.  Where a run ends is noted when its rows are sent for, so
// that adding up takes no look at the words; behind the last pair there are kBehind that are no words, so that a chunk's last step needs no bounds.
constexpr int kStep = 4;
template <typename T, typename TW, int LPT, int AHEAD>
__global__ void __launch_bounds__(256)
runs_kernel(const RunArgs a) {
  static_assert(AHEAD * kStep <= 32, "a bit for every row on its way");
  constexpr int E = kUnit<T>, NU = 8 / E, SLOT = kStep * NU * 256;     // units of a thread: eight columns
  extern __shared__ uint4 ring[];                        // [AHEAD][kStep][NU][256]
  pdl_wait();
  pdl_launch_dependents();
  const int64_t unit = (int64_t)blockIdx.x * (256 / LPT) + threadIdx.x / LPT;
  const int64_t c = unit / a.slices;
  if (c >= a.chunks) return;
  const int k0 = ((int)(unit - c * a.slices) * LPT * NU + threadIdx.x % LPT) * E;      // the first unit's column; the second is LPT units behind
  const int64_t lo = c * a.chunk;
  const int rows = (int)min((int64_t)a.chunk, a.T - lo), steps = (rows + kStep - 1) / kStep;
  const uint2* order = a.order + lo;
  const uint32_t ld = (uint32_t)a.lddy;
  const T* dY = (const T*)a.dY + k0;
  auto entries = [&](int step, uint4 (&e)[2]) {
    e[0] = reinterpret_cast<const uint4*>(order)[step * 2];
    e[1] = reinterpret_cast<const uint4*>(order)[step * 2 + 1];
  };
  uint4 now[2] = {}, next[2] = {};                                 // the pairs of the step to be sent for, and of the one behind it
  uint32_t ends = 0;                                     // four bits a slot: a run ends with this row
  auto fetch = [&](int step, int slot) {
    const uint32_t word[kStep + 1] = {now[0].x, now[0].z, now[1].x, now[1].z, next[0].x}, token[kStep] = {now[0].y, now[0].w, now[1].y, now[1].w};
    uint4* to = ring + slot * SLOT + threadIdx.x;
    uint32_t bits = 0;
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      const bool on = word[u] < a.V;
      const T* row = dY + (uint64_t)(on ? token[u] : 0) * ld;
#pragma unroll
      for (int q = 0; q < NU; ++q) copy_unit(to + (u * NU + q) * 256, row + q * LPT * E, on ? a.d - k0 - q * LPT * E : 0, a.vec);
      if (on && word[u + 1] != word[u]) bits |= 1u << u;
    }
    ends = (ends & ~(15u << (slot * kStep))) | bits << (slot * kStep);
    now[0] = next[0];
    now[1] = next[1];
    if (step + 2 < steps) entries(step + 2, next);
    else next[0] = *reinterpret_cast<const uint4*>(order + (step + 2) * kStep);          // for its first word
  };
  entries(0, now);
  if (steps > 1) entries(1, next);
  else next[0] = *reinterpret_cast<const uint4*>(order + kStep);
  bool open = lo > 0 && a.order[lo - 1].x == now[0].x;   // the run comes from before the chunk
#pragma unroll
  for (int s = 0; s < AHEAD; ++s) {
    if (s < steps) fetch(s, s);
    copies_commit();
  }
  uint64_t acc[NU][E / 2];
#pragma unroll
  for (int q = 0; q < NU; ++q)
#pragma unroll
    for (int j = 0; j < E / 2; ++j) acc[q][j] = 0;
  // what has been added up goes to the word's row, or to the chunk's place for the run that comes from before it or goes on behind it
  auto put = [&](uint32_t word, int part) {
#pragma unroll
    for (int q = 0; q < NU; ++q) {
      const int k = k0 + q * LPT * E, n = a.d - k;
      float f[E];
#pragma unroll
      for (int j = 0; j < E / 2; ++j) {
        const float2 w = unpack2(acc[q][j]);
        f[2 * j] = w.x;
        f[2 * j + 1] = w.y;
        acc[q][j] = 0;
      }
      if (n <= 0) continue;
      if (part < 0) {
        write_columns<TW, E>(a, word, k, n, f);
      } else {
        float* p = a.part + (c * 2 + part) * a.part_ld + k;
#pragma unroll
        for (int j = 0; j < E; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
      }
    }
  };
  int slot = 0;
  for (int s = 0; s < steps; ++s) {
    copies_wait<AHEAD - 1>();
    const uint4* at = ring + slot * SLOT + threadIdx.x;
    const uint32_t bits = ends >> (slot * kStep);
#pragma unroll
    for (int u = 0; u < kStep; ++u) {                    // rows that are not there are zeros
#pragma unroll
      for (int q = 0; q < NU; ++q) {
        uint64_t v[E / 2];
        unpack_unit<T>(at[(u * NU + q) * 256], v);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) acc[q][j] = add2(acc[q][j], v[j]);
      }
      if (bits >> u & 1) {
        put(order[s * kStep + u].x, open ? 0 : -1);
        open = false;
      }
    }
    if (s + AHEAD < steps) fetch(s + AHEAD, slot);
    copies_commit();
    slot = slot + 1 == AHEAD ? 0 : slot + 1;
  }
  const uint32_t last = order[rows - 1].x;
  if (last < a.V && order[rows].x == last) put(last, open ? 0 : 1);
}

// Warp w of block b looks at the end of chunk 8 b + w: where a run that began in that chunk goes over it, its parts (one for each chunk that it reaches) are added up,
// by the warp alone where they are few, by the eight warps of the block where they are many.  LPT lanes cover LPT * 8 columns (blockIdx.y: the rest); the
// groups of LPT lanes take runs of consecutive parts each, and their sums are added in a fixed order.
constexpr int kFewParts = 16;
template <typename TW, int LPT>
__global__ void __launch_bounds__(256)
joints_kernel(const RunArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int G = 32 / LPT;
  __shared__ float red[8][LPT][8];
  __shared__ int64_t many[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = lane / LPT, l = lane % LPT;
  const int k = (blockIdx.y * LPT + l) * 8, n = a.d - k;
  float acc[8];
  // parts [p0, p1) of a run that begins in chunk c: part 0 is its share of that chunk, part p its share of the p-th behind
  auto part_at = [&](int64_t c, int64_t p) { return reinterpret_cast<const float4*>(a.part + ((c + p) * 2 + (p == 0 ? 1 : 0)) * a.part_ld + k); };
  auto sum = [&](int64_t c, int64_t p0, int64_t p1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    if (n > 0) {
#pragma unroll 8
      for (int64_t p = p0; p < p1; ++p) {
        const float4 u = part_at(c, p)[0], v = part_at(c, p)[1];
        acc[0] += u.x; acc[1] += u.y; acc[2] += u.z; acc[3] += u.w;
        acc[4] += v.x; acc[5] += v.y; acc[6] += v.z; acc[7] += v.w;
      }
    }
#pragma unroll
    for (int o = LPT; o < 32; o <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
  };
  auto word_at = [&](int64_t i) { return i >= 0 && i < a.T ? a.order[i].x : kNoWord; };
  const int64_t c = (int64_t)blockIdx.x * 8 + warp, lo = c * a.chunk, hi = lo + a.chunk;
  // everything that most runs need is asked for at once: the words around, the words that the 32 chunks behind begin with, the first two parts
  const uint32_t word = word_at(hi - 1), next = word_at(hi), first = word_at(lo), prev = word_at(lo - 1);
  uint32_t begins = word_at((c + 1 + lane) * a.chunk);
  float4 two[4] = {};
  if (n > 0 && c + 1 < a.chunks) {
#pragma unroll
    for (int i = 0; i < 4; ++i) two[i] = part_at(c, i >> 1)[i & 1];
  }
  int64_t m = 0;                                         // parts
  if (word < a.V && next == word && !(first == word && prev == word)) {
    for (m = 1;; m += 32, begins = word_at((c + m + lane) * a.chunk)) {
      const unsigned on = __ballot_sync(0xffffffffu, begins == word);
      if (on == 0xffffffffu) continue;
      m += __ffs(~on) - 1;
      break;
    }
    if (m == 2) {
      if (group == 0 && n > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = reinterpret_cast<const float*>(two)[j] + reinterpret_cast<const float*>(two + 2)[j];
        write_columns<TW, 8>(a, word, k, n, acc);
      }
    } else if (m <= kFewParts * G) {
      const int64_t per = (m + G - 1) / G;
      sum(c, min(m, group * per), min(m, (group + 1) * per));
      if (group == 0 && n > 0) write_columns<TW, 8>(a, word, k, n, acc);
    }
  }
  if (lane == 0) many[warp] = m > kFewParts * G ? m : 0;
  __syncthreads();
  for (int w = 0; w < 8; ++w) {
    const int64_t parts = many[w], from = (int64_t)blockIdx.x * 8 + w;
    if (!parts) continue;
    const int64_t per = (parts + 8 * G - 1) / (8 * G), mine = warp * G + group;
    sum(from, min(parts, mine * per), min(parts, (mine + 1) * per));
    if (group == 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) red[warp][l][j] = acc[j];
    }
    __syncthreads();
    if (warp == 0 && group == 0 && n > 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
#pragma unroll
      for (int o = 0; o < 8; ++o)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += red[o][l][j];
      write_columns<TW, 8>(a, word_at((from + 1) * a.chunk - 1), k, n, acc);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- few tokens
// Eight tokens and 256 columns a block, a warp for each token: it looks through all words, lane j keeps which of the j-th 32 are its own (of the (j + 32)-th too, WORDS = 2), and the warp of the
// first token of a word lists the word's tokens and adds up their rows, U in flight; where they are many, the eight warps of the block do, an eighth of the list each, and
// their sums are added in order.  The blocks behind clear a range of dE's rows each, but for the words that occur, which they mark first.
constexpr int kFewTokens = 2048, kFewRows = 4096;        // bits that two words of 32 lanes hold; rows that a block can mark
template <typename T, typename TW, int WORDS>
__global__ void __launch_bounds__(256)
few_kernel(const RunArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int U = sizeof(T) == 2 ? 8 : 4, kAlone = 2 * U;
  constexpr int kTokens = 1024 * WORDS;
  __shared__ int32_t ids[kFewTokens];                    // kTokens of them; room for the sums of eight warps
  __shared__ uint16_t list[8][kTokens];
  __shared__ int2 many[8];                               // a word that all warps add up, and how many tokens it has
  float(*red)[32][8] = reinterpret_cast<float(*)[32][8]>(ids);           // once the words have been looked through
  static_assert(sizeof(ids) >= 8 * 32 * 8 * sizeof(float), "");
  uint32_t* marks = reinterpret_cast<uint32_t*>(list);
  static_assert(kFewRows / 8 <= (int)sizeof(list), "");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_tokens = (int)a.T;
  if ((int)blockIdx.x >= a.token_blocks) {
    const int64_t first = (int64_t)(blockIdx.x - a.token_blocks) * a.clear_rows;
    const int rows = (int)min((int64_t)a.clear_rows, a.clear.rows - first);
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += 256) marks[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < n_tokens; t += 256) {
      const int64_t r = (int64_t)a.ids[t] - first;
      if (r >= 0 && r < rows) atomicOr(marks + (r >> 5), 1u << (r & 31));
    }
    __syncthreads();
    clear_rows(a.clear.p + first * a.clear.pitch, rows, a.clear, threadIdx.x, 256, [&](int64_t r) { return (marks[r >> 5] >> (r & 31)) & 1; });
    return;
  }
#pragma unroll
  for (int i = threadIdx.x; i < kTokens; i += 256) ids[i] = i < n_tokens ? a.ids[i] : -1;
  __syncthreads();
  const int eight = blockIdx.x / a.slices, t = eight * 8 + warp, k = (((int)blockIdx.x - eight * a.slices) * 32 + lane) * 8, n = a.d - k;
  const int32_t word = t < n_tokens ? ids[t] : -1;
  uint32_t mine[WORDS] = {};
  bool first = word >= 0 && (uint32_t)word < a.V;
  for (int j = 0; first && j * 32 < n_tokens; j += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t m = __ballot_sync(0xffffffffu, ids[(j + u) * 32 + lane] == word);
      if (lane == ((j + u) & 31)) mine[WORDS == 1 ? 0 : (j + u) >> 5 & 1] = m;
      const int at = (j + u) * 32;
      if (at <= t && (at + 32 <= t ? m : m & ((1u << (t - at)) - 1))) first = false;
    }
  }
  int count = 0;
  if (first) {
#pragma unroll
    for (int h = 0; h < WORDS; ++h) {
      int inc = __popc(mine[h]);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      int at = count + inc - __popc(mine[h]);
      for (uint32_t m = mine[h]; m; m &= m - 1) list[warp][at++] = (uint16_t)((h * 32 + lane) * 32 + __ffs(m) - 1);
      count += __shfl_sync(0xffffffffu, inc, 31);
    }
    __syncwarp();
  }
  float acc[8];
  auto sum = [&](const uint16_t* tokens, int p0, int p1) {
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q] = 0.f;
    for (int p = p0; p < p1; p += U) {
      Raw8<T> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = p + u < p1 ? tokens[p + u] : 0;
        raw[u] = load8((const T*)a.dY + (int64_t)at * a.lddy + k, p + u < p1 ? n : 0, a.vec, at + 1 < n_tokens);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u < p1) {
          float v[8];
          unpack8(raw[u], n, v);
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[q] += v[q];
        }
      }
    }
  };
  if (count > 0 && count <= kAlone) {
    sum(list[warp], 0, count);
    if (n > 0) write_columns<TW, 8>(a, (uint32_t)word, k, n, acc);
  }
  if (lane == 0) many[warp] = make_int2(word, count > kAlone ? count : 0);
  __syncthreads();
  for (int w = 0; w < 8; ++w) {
    const int tokens = many[w].y, per = (tokens + 7) / 8;
    if (!tokens) continue;
    sum(list[w], min(tokens, warp * per), min(tokens, (warp + 1) * per));
#pragma unroll
    for (int q = 0; q < 8; ++q) red[warp][lane][q] = acc[q];
    __syncthreads();
    if (warp == 0 && n > 0) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        acc[q] = 0.f;
#pragma unroll
        for (int o = 0; o < 8; ++o) acc[q] += red[o][lane][q];
      }
      write_columns<TW, 8>(a, (uint32_t)many[w].x, k, n, acc);
    }
    __syncthreads();
  }
}

}  // namespace emb
}  // namespace flop
